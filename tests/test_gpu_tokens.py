"""Token caches on the GPU against plain 64-bit forms: writing and reading cells (as they are and as
e4m3 codes with power-of-two scales), attention of chunks and single tokens over pages with and
without a window and sinks, and the calls' refusals.

Tolerances, fixed by the arithmetic: a value that is only copied is equal bit for bit, and so is a
quantised one (its scaling is exact and its one rounding is defined).  An attention output has
  u |out| (its own rounding, u the unit of its type) + u A (the probabilities' rounding to the
  type, A = sum p |v|) + c A, c = 2^-24 (8 sqrt(D) E + 8 sqrt(n) + 64)
with E the row's largest sum of |q k| times the scale: rounding errors of a score's D products and
of the sums over n cells at eight times their random-walk size, and 64 units for the exponential.
A log-sum is off by c (1 + |lse|)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def M():
    from paper_2607_18582_gb300 import build
    build.build()
    from paper_2607_18582_gb300 import mure
    return mure


@pytest.fixture(scope="module")
def ctx(M):
    return M.mure_create(0)


TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def codes_of(x):
    """(codes, scale bytes) of rows in 64 bits, from the definition."""
    x = x.double().cpu()
    a = x.abs().amax(-1)
    bad = ~torch.isfinite(x).all(-1)
    e = torch.full(a.shape, -127, dtype=torch.int64)
    for k in range(-127, 128):                     # the least k with a 2^-k <= 448
        e = torch.where(a * 2.0 ** -(k - 1) > 448.0, torch.full_like(e, k), e) if k > -127 else e
    e = torch.where(bad, torch.zeros_like(e), e)
    y = torch.where(bad[..., None], torch.zeros_like(x), x) * torch.pow(2.0, -e.double())[..., None]
    # every e4m3 magnitude, and the nearest one (ties to the even code)
    mags = torch.tensor([(m / 8.0) * 2.0 ** -6 if ex == 0 else (1 + m / 8.0) * 2.0 ** (ex - 7)
                         for ex in range(16) for m in range(8)][:127], dtype=torch.float64)
    flat = y.abs().reshape(-1)
    hi = torch.searchsorted(mags, flat).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dh, dl = (mags[hi] - flat).abs(), (mags[lo] - flat).abs()
    code = torch.where(dl < dh, lo, torch.where(dl > dh, hi, torch.where(lo % 2 == 0, lo, hi)))
    code = (code + 128 * (torch.signbit(y).reshape(-1))).to(torch.uint8).view(y.shape)
    return code, torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)


def values_of(code, byte):
    code, byte = code.cpu().to(torch.int64), byte.cpu().to(torch.int64)
    ex, m = (code >> 3) & 15, code & 7
    mag = torch.where(ex == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * torch.pow(2.0, (ex - 7).double()))
    v = torch.where(code >= 128, -mag, mag) * torch.pow(2.0, (byte - 127).double())[..., None]
    return torch.where((byte == 255)[..., None], torch.full_like(v, math.nan), v)


class Batch:
    """Sequences with their pages, pools with content, and the new tokens' rows."""

    def __init__(self, M, ctx, new, pos, kv, heads, hk, d, page, dtype, form, seed=0, window=0, sinks=0, scale=0.0,
                 spare=2, table=None, gain=1.0):
        self.M, self.ctx = M, ctx
        self.new, self.pos, self.kv = list(new), list(pos), list(kv)
        self.heads, self.hk, self.d, self.page, self.dtype, self.form = heads, hk, d, page, dtype, form
        self.window, self.sinks, self.scale = window, sinks, scale
        g = torch.Generator(device="cuda").manual_seed(seed)
        need = [-(-k // page) for k in self.kv]
        self.n_pages = sum(need) + spare
        if table is None:
            order = np.random.default_rng(seed).permutation(self.n_pages)
            table = np.full((len(kv), max(need + [1])), -7, np.int32)     # unused entries are not read
            at = 0
            for b, k in enumerate(need):
                table[b, :k] = order[at:at + k]
                at += k
        self.table = table
        dt = TYPES[dtype]
        shape = (self.n_pages, hk, page, d)
        x = [torch.randn(shape, generator=g, device="cuda") * gain for _ in range(2)]
        if form == "e4m3":
            pairs = [codes_of(t) for t in x]
            self.pools = [p[0].cuda().view(torch.float8_e4m3fn) for p in pairs] + [p[1].cuda() for p in pairs]
        else:
            self.pools = [t.to(dt) for t in x]
        total = sum(self.new)
        self.q = (torch.randn(total, heads, d, generator=g, device="cuda") * 2).to(dt)
        self.k = torch.randn(total, hk, d, generator=g, device="cuda").to(dt)
        self.v = torch.randn(total, hk, d, generator=g, device="cuda").to(dt)
        self.cache = M.mure_tokens_create(ctx, hk, d, page, self.n_pages, dtype=dtype, form=form, buffers=tuple(self.pools))
        self.plan = self.make_plan()

    def make_plan(self, plan=None):
        return self.M.mure_tokens_plan(self.cache, self.heads, self.new, self.pos, self.kv, self.table, window=self.window,
                                       sinks=self.sinks, scale=self.scale, plan=plan)

    def dense(self, which, b):
        """Cells of sequence b in 64 bits, [kv][hk][d]."""
        ids = torch.from_numpy(self.table[b, :-(-self.kv[b] // self.page)].astype(np.int64))
        pool = self.pools[which]
        if self.form == "e4m3":
            x = values_of(pool.view(torch.uint8)[ids.cuda()], self.pools[2 + which][ids.cuda()])
        else:
            x = pool[ids.cuda()].double().cpu()
        return x.transpose(1, 2).reshape(-1, self.hk, self.d)[:self.kv[b]].cuda()

    def reference(self):
        """out, lse, and the tolerances of both, in 64 bits: masked cells take no part whatever they hold."""
        outs, lses, tols, ltols, row, grp = [], [], [], [], 0, self.heads // self.hk
        scale, u = self.scale or self.d ** -0.5, UNIT[self.dtype]
        for b, n in enumerate(self.new):
            if n == 0:
                continue
            k, v = self.dense(0, b), self.dense(1, b)
            q = self.q[row:row + n].double()
            row += n
            at = torch.arange(self.pos[b], self.pos[b] + n, device="cuda")[:, None]
            cell = torch.arange(self.kv[b], device="cuda")[None]
            see = cell <= at
            if self.window:
                see = see & ((cell > at - self.window) | (cell < self.sinks))
            out = torch.zeros(n, self.heads, self.d, dtype=torch.float64, device="cuda")
            lse = torch.full((n, self.heads), -math.inf, dtype=torch.float64, device="cuda")
            tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
            if self.kv[b]:
                for h in range(self.heads):
                    kk, vv = k[:, h // grp], v[:, h // grp]
                    s = torch.where(see, q[:, h] @ kk.nan_to_num(0, 0, 0).T * scale, torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
                    badk = (~torch.isfinite(kk)).any(-1)
                    s = torch.where(see & badk[None], torch.full_like(s, math.nan), s)
                    lse[:, h] = torch.logsumexp(s, -1)
                    p = torch.where(see, torch.exp(s - lse[:, h:h + 1]), torch.zeros_like(s))
                    bad = (~torch.isfinite(vv)).double()
                    out[:, h] = p @ vv.nan_to_num(0, 0, 0)
                    A = p @ vv.nan_to_num(0, 0, 0).abs()
                    out[:, h] = torch.where((see.double() @ bad) > 0, torch.full_like(A, math.nan), out[:, h])
                    E = torch.where(see, q[:, h].abs() @ kk.nan_to_num(0, 0, 0).abs().T * scale, torch.zeros_like(s)).amax(-1)
                    c = 2.0 ** -24 * (8 * math.sqrt(self.d) * E + 8 * math.sqrt(self.kv[b]) + 64)
                    tol[:, h] = u * out[:, h].abs() + (u + c[:, None]) * A + 1e-30
                    ltol[:, h] = c * (1 + lse[:, h].abs())
                empty = ~see.any(-1)
                out[empty], lse[empty], tol[empty] = 0.0, -math.inf, 0.0
            outs.append(out); lses.append(lse); tols.append(tol); ltols.append(ltol)
        if not outs:
            return (torch.zeros(0, self.heads, self.d, device="cuda"),) * 2 + (torch.zeros(0, self.heads, device="cuda"),) * 2
        return torch.cat(outs), torch.cat(tols), torch.cat(lses), torch.cat(ltols)

    def check(self, got=None):
        out, lse = got if got is not None else self.M.mure_tokens_attend(self.cache, self.plan, self.q, lse=True)
        self.M.mure_synchronize(self.ctx)
        ref, tol, rlse, ltol = self.reference()
        bad = torch.isnan(ref)
        assert torch.equal(torch.isnan(out), bad)
        err = (out.double() - ref).abs()
        assert bool(((err <= tol) | bad).all()), (float((err - tol)[~bad].max()), float(err[~bad].max()))
        inf = torch.isinf(rlse)
        assert torch.equal(torch.isinf(lse), inf) and bool((lse[inf] < 0).all())
        off = (lse.double() - rlse).abs()
        ok = (off <= ltol) | inf | torch.isnan(rlse)
        assert bool(ok.all()), float(off[~inf].max())
        return out, lse


# ------------------------------------------------------------------ cells --

SHAPES = [(8, 128, 16), (1, 64, 8), (3, 40, 32), (2, 256, 64), (5, 8, 128), (2, 96, 1024)]


@pytest.mark.parametrize("form", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("hk,d,page", SHAPES)
def test_append_and_read(M, ctx, dtype, form, hk, d, page):
    """Cells equal the definition bit for bit, other cells keep their content, and reading gives the
    values back; zero-length and odd sequences, chunks that start and end inside pages."""
    new, pos = [1, 0, 37, 5, 130, 0, 16], [0, 9, 3, 2 * page - 2, 100, 0, 16]
    kv = [a + b for a, b in zip(new, pos)]
    kv[3] += 11                                   # cells past the new ones
    t = Batch(M, ctx, new, pos, kv, hk, hk, d, page, dtype, form, seed=d + page)
    before = [p.clone() for p in t.pools]
    M.mure_tokens_append(t.cache, t.plan, t.k, t.v)
    got_new = M.mure_tokens_read(t.cache, t.plan, new=True)
    got_all = M.mure_tokens_read(t.cache, t.plan)
    M.mure_synchronize(ctx)
    ids = np.concatenate([t.table[b, (np.arange(p, p + n)) // page] for b, (n, p) in enumerate(zip(new, pos))])
    slots = np.concatenate([np.arange(p, p + n) % page for n, p in zip(new, pos)])
    ids, slots = torch.from_numpy(ids.astype(np.int64)).cuda(), torch.from_numpy(slots).cuda()
    for w, x in enumerate((t.k, t.v)):
        want = before[w].clone()
        if form == "e4m3":
            code, byte = codes_of(x)
            scale = before[2 + w].clone()
            want.view(torch.uint8)[ids, :, slots] = code.cuda()
            scale[ids, :, slots] = byte.cuda()
            assert torch.equal(t.pools[2 + w], scale)
            assert torch.equal(t.pools[w].view(torch.uint8), want.view(torch.uint8))
            back = values_of(code, byte).to(TYPES[dtype]).cuda()
        else:
            want[ids, :, slots] = x
            assert torch.equal(t.pools[w], want)
            back = x
        assert torch.equal(got_new[w], back)
        dense = torch.cat([t.dense(w, b) for b in range(len(kv))]).to(TYPES[dtype])
        assert torch.equal(got_all[w], dense)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_quantised_edges(M, ctx, dtype):
    """Rows of zeros, of subnormals, at and around the scale's steps, of the type's largest values;
    a row with an infinity or a NaN reads as NaN and leaves its neighbours alone."""
    d, dt = 16, TYPES[dtype]
    fi = torch.finfo(dt)
    rows = [torch.zeros(d), torch.full((d,), float(fi.tiny)), torch.full((d,), float(fi.max)), torch.full((d,), -float(fi.max))]
    if dtype != "f16":
        rows += [torch.full((d,), 2.0 ** -133), torch.full((d,), 1.75 * 2.0 ** -119)]
    for a in (448.0, 449.0 if dtype == "f32" else 450.0, 1.75, 1.7578125, 0.875, 1.0, 2.0 ** 10):
        rows.append(torch.linspace(-a, a, d))
    rows.append(torch.tensor([17.0, 18, 19, 21, 23, 25, 27, 29, 2 ** -6, 2 ** -9, 2 ** -10, 3 * 2 ** -10, 2 ** -11, 448, 0, -0.0]))
    for bad in (math.inf, -math.inf, math.nan):
        r = torch.ones(d)
        r[5] = bad
        rows.append(r)
    x = torch.stack(rows).to(dt).cuda()[:, None]
    n = len(rows)
    t = Batch(M, ctx, [n], [0], [n], 1, 1, d, 8, dtype, "e4m3")
    M.mure_tokens_append(t.cache, t.plan, x, x.flip(0))
    k, v = M.mure_tokens_read(t.cache, t.plan)
    for got, src in ((k, x), (v, x.flip(0))):
        want = values_of(*codes_of(src)).to(dt).cuda()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got.nan_to_num(0), want.nan_to_num(0))
        assert torch.equal(torch.isnan(got).any(-1), ~torch.isfinite(src).all(-1))


@pytest.mark.parametrize("form", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_any_stride(M, ctx, dtype, form):
    """Inputs and outputs that are slices: columns of one projection's output, heads before tokens,
    rows that start off a 16-byte boundary."""
    hk, d, n = 3, 24, 21
    t = Batch(M, ctx, [n], [4], [n + 4], 6, hk, d, 16, dtype, form)
    M.mure_tokens_append(t.cache, t.plan, t.k, t.v)
    want = [x.clone() for x in M.mure_tokens_read(t.cache, t.plan, new=True)]
    ref = M.mure_tokens_attend(t.cache, t.plan, t.q).clone()
    for p in t.pools:
        p.view(torch.uint8).zero_()
    fused = torch.zeros(n, 12 * d + 5, dtype=TYPES[dtype], device="cuda")
    view = fused[:, 1:1 + 12 * d].unflatten(1, (12, d))
    view[:, :6], view[:, 6:9], view[:, 9:] = t.q, t.k, t.v
    M.mure_tokens_append(t.cache, t.plan, view[:, 6:9], view[:, 9:])
    outs = [torch.zeros(hk, n, d + 3, dtype=TYPES[dtype], device="cuda")[..., 2:2 + d].transpose(0, 1) for _ in range(2)]
    M.mure_tokens_read(t.cache, t.plan, new=True, out=tuple(outs))
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    big = torch.full((n, 6, 2 * d + 1), 3.0, dtype=TYPES[dtype], device="cuda")
    out = big[..., 1:1 + d]
    t2 = Batch(M, ctx, [n], [4], [n + 4], 6, hk, d, 16, dtype, form)      # the first four cells' content again
    M.mure_tokens_append(t2.cache, t2.plan, t.k, t.v)
    M.mure_tokens_attend(t2.cache, t2.plan, view[:, :6], out=out)
    assert torch.equal(out, ref)
    assert bool((big[..., 0] == 3).all()) and bool((big[..., 1 + d:] == 3).all())


# -------------------------------------------------------------- attention --

HEADS = [(8, 2, 64, 16), (4, 4, 128, 8), (32, 8, 128, 64), (5, 1, 40, 32), (24, 2, 80, 16), (2, 1, 256, 16), (48, 1, 96, 128),
         (3, 3, 8, 1024)]
RAGGED = [([1, 1, 1, 1, 1], [0, 1, 15, 500, 1300]),                       # one token each
          ([3, 0, 1, 17, 40], [5, 7, 0, 33, 256]),                        # small chunks, a sequence without new tokens
          ([200, 1, 129, 64], [0, 900, 77, 640])]                         # long chunks beside a single token


@pytest.mark.parametrize("form", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("new,past", RAGGED)
@pytest.mark.parametrize("heads,hk,d,page", HEADS)
def test_attend(M, ctx, heads, hk, d, page, new, past, dtype, form):
    Batch(M, ctx, new, past, [a + b for a, b in zip(new, past)], heads, hk, d, page, dtype, form, seed=7).check()


@pytest.mark.parametrize("form", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (100, 0), (129, 130), (5000, 3), (7, 2000)])
@pytest.mark.parametrize("new,past", RAGGED[:1] + RAGGED[2:])
def test_attend_window_and_sinks(M, ctx, window, sinks, new, past, dtype, form):
    Batch(M, ctx, new, past, [a + b for a, b in zip(new, past)], 8, 2, 64, 16, dtype, form, seed=3, window=window,
          sinks=sinks).check()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [64, 128])
def test_rows_without_cells(M, ctx, dtype, d):
    """No cells held; positions so far past the cells that a window leaves none; sinks alone; fewer
    cells than positions."""
    new, pos, kv = [4, 3, 200, 9, 2, 1], [0, 90, 400, 20, 0, 5000], [0, 40, 300, 0, 1, 7]
    for window, sinks in ((0, 0), (32, 0), (32, 2), (150, 0)):
        Batch(M, ctx, new, pos, kv, 4, 2, d, 16, dtype, "same", window=window, sinks=sinks).check()


@pytest.mark.parametrize("dtype,form", [("bf16", "same"), ("f16", "e4m3")])
def test_many_chunks_of_all_lengths(M, ctx, dtype, form):
    """More pieces of work than blocks, short ones (one tile of rows) before and after long ones."""
    rng = np.random.default_rng(5)
    new = [int(x) for x in rng.integers(1, 150, 300)]
    past = [int(x) for x in rng.integers(0, 1500, 300)]
    t = Batch(M, ctx, new, past, [a + b for a, b in zip(new, past)], 12, 4, 64, 32, dtype, form)
    for _ in range(3):
        t.check()


@pytest.mark.parametrize("scale", [1.0, 0.01, 3.0])
def test_scale(M, ctx, scale):
    Batch(M, ctx, [70, 1], [40, 300], [110, 301], 4, 2, 64, 16, "bf16", "same", scale=scale).check()


@pytest.mark.parametrize("form", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("new,past,window,sinks", [([1, 1], [700, 90], 0, 0), ([150, 2], [300, 50], 0, 0),
                                                  ([1, 140], [900, 500], 64, 3)])
def test_masked_cells_never_reach_an_output(M, ctx, new, past, window, sinks, dtype, form):
    """NaN and infinities in every cell that no row may attend to, and at later cells of a chunk: rows
    that do not see them keep their values, rows that do are NaN."""
    kv = [a + b for a, b in zip(new, past)]
    t = Batch(M, ctx, new, past, kv, 8, 2, 64, 16, dtype, form, window=window, sinks=sinks)
    held = torch.zeros(t.n_pages, t.page, dtype=torch.bool)
    for b, (p, k) in enumerate(zip(past, kv)):
        for j in range(k):
            if not window or j > p - window or j < sinks:
                held[t.table[b, j // t.page], j % t.page] = True
    dead = (~held)[:, None].expand(-1, t.hk, -1).cuda()
    if form == "e4m3":
        t.pools[2][dead] = 255
        t.pools[3][dead] = 255
        t.pools[0].view(torch.uint8)[dead] = 0x7F
        t.pools[1].view(torch.uint8)[dead] = 0xFF
    else:
        t.pools[0][dead] = math.nan
        t.pools[1][dead] = math.inf
    out, _ = t.check()
    assert bool(torch.isfinite(out).all())
    b = int(np.argmax(new))                       # now a late cell of the longest chunk: its own row and later see it
    j = kv[b] - max(1, new[b] // 3)
    page, slot = int(t.table[b, j // t.page]), j % t.page
    for w, val in ((1, math.nan), (0, math.nan)):
        if form == "e4m3":
            t.pools[2 + w][page, 0, slot] = 255
        else:
            t.pools[w][page, 0, slot] = val
            if dtype == "f32":                     # (the bits that the GPU's own arithmetic gives)
                t.pools[w].view(torch.int32)[page, 0, slot, ::2] = 0x7FFFFFFF
                t.pools[w].view(torch.int32)[page, 0, slot, 1::2] = -1
        out, _ = t.check()
        bad = torch.isnan(out).any(-1)
        row0 = sum(new[:b])
        seen = torch.arange(new[b]) + past[b] >= j
        assert torch.equal(bad[row0:row0 + new[b], 0].cpu(), seen) and not bool(bad[:, 4:].any())


def test_scores_at_the_ends_of_the_range(M, ctx):
    """Scores of thousands, equal scores, and one cell that outweighs all others."""
    for dtype in TYPES:
        t = Batch(M, ctx, [1, 130], [600, 400], [601, 530], 4, 2, 64, 16, dtype, "same", scale=1.0)
        t.pools[0].zero_()
        t.check()                                  # equal scores: the mean of the cells
        page, slot = int(t.table[1, 3]), 5
        t.pools[0][page, :, slot] = 40.0
        t.q.fill_(3.0)
        t.check()
        t.pools[0].neg_()
        t.check()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [64, 128, 256])
def test_scales_of_all_sizes(M, ctx, dtype, d):
    """e4m3 rows whose scales differ by up to 2^20 within a sequence, rows of zeros and of the least scale
    beside large ones, and queries of very small and very large magnitude (f16: as far as it goes)."""
    lo, hi = (-10, 10) if dtype != "f16" else (-6, 4)
    t = Batch(M, ctx, [1, 90], [700, 300], [701, 390], 8, 2, d, 16, dtype, "e4m3", seed=9)
    g = torch.Generator(device="cuda").manual_seed(1)
    for w, middle in ((2, 113), (3, 119)):         # (of K smaller: scores stay within tens)
        e = torch.randint(lo, hi + 1, t.pools[w].shape, generator=g, device="cuda")
        t.pools[w].copy_((middle + e).to(torch.uint8))
        pick = torch.rand(t.pools[w].shape, generator=g, device="cuda")
        t.pools[w][pick < 0.05] = 0                # least scale, codes of any size
        t.pools[w - 2].view(torch.uint8)[pick > 0.95] = 0
    t.check()
    if dtype != "f16":
        t.q.mul_(2.0 ** -60)
        t.check()
        t.q.mul_(2.0 ** 90)
        t.pools[2][t.pools[2] > 40] -= 40
        t.check()
    else:
        t.q[..., ::2].mul_(2.0 ** -12)
        t.check()


@pytest.mark.parametrize("new", [1, 100])
def test_largest_f16_values_as_codes(M, ctx, new):
    """f16 values whose nearest code stands for 65,536: attention takes them as finite."""
    t = Batch(M, ctx, [new], [60], [60 + new], 2, 1, 64, 16, "f16", "e4m3")
    big = torch.full((60, 1, 64), 65504.0, device="cuda", dtype=torch.float16)
    big[::2] = -60000.0
    plan = M.mure_tokens_plan(t.cache, 2, [60], [0], [60], t.table)
    M.mure_tokens_append(t.cache, plan, big * 2.0 ** -20, big)
    out, _ = t.check()
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("dtype,form", [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same")])
def test_offsets_past_32_bits(M, ctx, dtype, form):
    """Pages at the far end of pools of more than 2^31 values."""
    hk, d, page = 8, 128, 64
    n_pages = 2 ** 31 // (hk * d * page) + 40
    t = Batch(M, ctx, [150, 1], [100, 300], [250, 301], 16, hk, d, page, dtype, form)
    if form == "same":
        big = [torch.empty(n_pages, hk, page, d, dtype=TYPES[dtype], device="cuda") for _ in range(2)]
    else:
        big = [torch.empty(n_pages, hk, page, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
        big += [torch.empty(n_pages, hk, page, dtype=torch.uint8, device="cuda") for _ in range(2)]
    shift = n_pages - t.n_pages
    for b, s in zip(big, t.pools):
        b.view(torch.uint8)[shift:] = s.view(torch.uint8) if s.dtype != torch.uint8 else s
    far = M.mure_tokens_create(ctx, hk, d, page, n_pages, dtype=dtype, form=form, buffers=tuple(big))
    plan = M.mure_tokens_plan(far, 16, t.new, t.pos, t.kv, np.where(t.table >= 0, t.table + shift, 0))
    M.mure_tokens_append(t.cache, t.plan, t.k, t.v)
    M.mure_tokens_append(far, plan, t.k, t.v)
    for a, b in zip(M.mure_tokens_read(t.cache, t.plan), M.mure_tokens_read(far, plan)):
        assert torch.equal(a, b)
    out, lse = M.mure_tokens_attend(far, plan, t.q, lse=True)
    t.check((out, lse))


def test_long_axis(M, ctx):
    """One row over a long axis, split and joined, in every form."""
    for dtype, form in (("bf16", "same"), ("f16", "e4m3"), ("f32", "same"), ("f32", "e4m3"), ("bf16", "e4m3")):
        Batch(M, ctx, [1, 40], [40001, 20000], [40002, 20040], 4, 1, 64, 64, dtype, form).check()


def test_shared_pages(M, ctx):
    """Sequences over the same pages (mutants that share the original's cells): each as if alone."""
    t = Batch(M, ctx, [30], [200], [230], 8, 2, 64, 16, "bf16", "same")
    alone = M.mure_tokens_attend(t.cache, t.plan, t.q)
    plan = M.mure_tokens_plan(t.cache, 8, [30] * 5, [200] * 5, [230] * 5, np.repeat(t.table, 5, 0))
    q = t.q.repeat(5, 1, 1)
    many = M.mure_tokens_attend(t.cache, plan, q).view(5, 30, 8, 64)
    ref, tol, _, _ = t.reference()
    for i in range(5):
        assert bool(((many[i].double() - ref).abs() <= tol).all())
    assert bool(((alone.double() - ref).abs() <= tol).all())
    with pytest.raises(M.MureError) as ei:         # ... but they cannot all write them
        M.mure_tokens_append(t.cache, plan, t.k.repeat(5, 1, 1), t.v.repeat(5, 1, 1))
    assert ei.value.status == 1 and "cell" in str(ei.value)


def test_equal_calls_give_equal_bits_and_plans_are_reused(M, ctx):
    for dtype, form in (("bf16", "same"), ("f16", "e4m3"), ("f32", "same")):
        t = Batch(M, ctx, [1, 300, 2], [9000, 1000, 50], [9001, 1300, 52], 8, 2, 128, 16, dtype, form)
        first = [x.clone() for x in M.mure_tokens_attend(t.cache, t.plan, t.q, lse=True)]
        for _ in range(5):
            again = M.mure_tokens_attend(t.cache, t.plan, t.q, lse=True)
            assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
        # another batch in the same plan, then the first again
        new, pos, kv = t.new, t.pos, t.kv
        t.new, t.pos, t.kv = [303, 0, 0], [8000, 0, 1], [8303, 5, 9]
        t.make_plan(t.plan)
        t.check()
        t.new, t.pos, t.kv = new, pos, kv
        t.make_plan(t.plan)
        again = M.mure_tokens_attend(t.cache, t.plan, t.q, lse=True)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


def test_another_stream_and_the_library_s_own_pools(M):
    """A context on a stream of its own, called from torch's current stream; pools that the library
    allocates start with zeros."""
    for torch_allocator in (True, False):
        ctx = M.mure_create(0, stream=torch.cuda.Stream(), torch_allocator=torch_allocator)
        c = M.mure_tokens_create(ctx, 2, 64, 16, 40, dtype="bf16")
        plan = M.mure_tokens_plan(c, 4, [300], [0], [300], np.arange(40, dtype=np.int32)[None])
        k, v = M.mure_tokens_read(c, plan)
        assert not bool(k.any()) and not bool(v.any())
        for i in range(20):
            x = torch.full((300, 2, 64), float(i), device="cuda", dtype=torch.bfloat16)
            y = x + 1
            M.mure_tokens_append(c, plan, x, y)
            del x
            junk = torch.full((300, 2, 64), -1.0, device="cuda", dtype=torch.bfloat16)
            k, v = M.mure_tokens_read(c, plan)
            q = torch.ones(300, 4, 64, device="cuda", dtype=torch.bfloat16)
            o = M.mure_tokens_attend(c, plan, q)
            assert bool((k == i).all()) and bool((v == i + 1).all())
            assert bool((o == i + 1).all()), i
            del junk
        M.mure_synchronize(ctx)


def test_no_work(M, ctx):
    t = Batch(M, ctx, [0, 0], [0, 3], [0, 7], 4, 2, 64, 16, "bf16", "same")
    assert M.mure_tokens_attend(t.cache, t.plan, t.q).shape == (0, 4, 64)
    M.mure_tokens_append(t.cache, t.plan, t.k, t.v)
    k, v = M.mure_tokens_read(t.cache, t.plan, new=True)
    assert k.shape[0] == 0
    plan = M.mure_tokens_plan(t.cache, 4, [], [], [], np.zeros((0, 1), np.int32))
    assert M.mure_tokens_read(t.cache, plan)[0].shape[0] == 0
    M.mure_synchronize(ctx)


# --------------------------------------------------------------- refusals --

def test_create_refusals(M, ctx):
    import ctypes as C
    ok = dict(n_kv_heads=2, head_dim=64, page_size=16, dtype=2, form=0, reserved=0, n_pages=4, k=None, v=None,
              k_scale=None, v_scale=None)
    cases = [dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=0), dict(head_dim=12), dict(head_dim=264),
             dict(page_size=4), dict(page_size=24), dict(page_size=2048), dict(n_pages=0), dict(n_pages=2 ** 31),
             dict(reserved=1), dict(k=4096), dict(k=4096, v=4104), dict(k=4096, v=4096, k_scale=4096),
             dict(form=1, k=4096, v=4096, k_scale=4096)]
    for bad, status in [(c, 1) for c in cases] + [(dict(dtype=3), 2), (dict(form=2), 2)]:
        d = M._TokensDesc(**{**ok, **bad})
        out = C.c_void_p(77)
        assert M.lib().mure_tokens_create(ctx.h, C.byref(d), C.byref(out)) == status, bad
        assert not out.value and M.lib().mure_last_error(ctx.h)
    d = M._TokensDesc(**ok)
    assert M.lib().mure_tokens_create(ctx.h, None, C.byref(C.c_void_p())) == 1
    assert M.lib().mure_tokens_create(ctx.h, C.byref(d), None) == 1
    assert M.lib().mure_tokens_create(None, C.byref(d), C.byref(C.c_void_p())) == 1


def test_plan_refusals(M, ctx):
    t = Batch(M, ctx, [2], [14], [16], 4, 2, 64, 16, "bf16", "same")

    def plan(heads=4, new=(2,), pos=(14,), kv=(16,), table=((0,),), **kw):
        return M.mure_tokens_plan(t.cache, heads, list(new), list(pos), list(kv), np.array(table, np.int32), **kw)

    plan()
    for bad in (dict(heads=3), dict(heads=0), dict(new=(-1,)), dict(pos=(-1,)), dict(kv=(-1,)), dict(kv=(17,)),
                dict(table=((-1,),)), dict(table=((t.n_pages,),)), dict(window=-1), dict(sinks=2),
                dict(window=3, sinks=-1), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf),
                dict(pos=(2 ** 30,))):
        with pytest.raises(M.MureError) as ei:
            plan(**bad)
        assert ei.value.status == 1, bad
    with pytest.raises(ValueError):
        plan(new=(1, 2))
    # a plan whose new batch was refused holds none
    p = plan()
    with pytest.raises(M.MureError):
        M.mure_tokens_plan(t.cache, 3, [2], [14], [16], np.zeros((1, 1), np.int32), plan=p)
    with pytest.raises(M.MureError) as ei:
        M.mure_tokens_attend(t.cache, p, t.q)
    assert ei.value.status == 1


def test_call_refusals(M, ctx):
    import ctypes as C
    t = Batch(M, ctx, [2], [14], [16], 4, 2, 64, 16, "bf16", "same")
    before = [p.clone() for p in t.pools]
    L, rows = M.lib(), M._TokensRows
    good = rows(t.k.data_ptr(), t.k.stride(0), t.k.stride(1))
    qrow = rows(t.q.data_ptr(), t.q.stride(0), t.q.stride(1))
    out = torch.zeros_like(t.q)
    orow = rows(out.data_ptr(), out.stride(0), out.stride(1))
    null, odd = rows(None, 128, 64), rows(t.k.data_ptr() + 1, 128, 64)
    same = rows(out.data_ptr(), 0, 64)
    r = C.byref
    assert L.mure_tokens_append(t.cache.h, None, r(good), r(good)) == 1
    assert L.mure_tokens_append(None, t.plan.h, r(good), r(good)) == 1
    for a, b in ((null, good), (good, null), (odd, good)):
        assert L.mure_tokens_append(t.cache.h, t.plan.h, r(a), r(b)) == 1
        assert L.mure_tokens_read(t.cache.h, t.plan.h, 1, r(a), r(b)) == 1
    assert L.mure_tokens_append(t.cache.h, t.plan.h, None, r(good)) == 1
    assert L.mure_tokens_read(t.cache.h, t.plan.h, 2, r(good), r(good)) == 1
    assert L.mure_tokens_attend(t.cache.h, t.plan.h, r(null), r(orow), None) == 1
    assert L.mure_tokens_attend(t.cache.h, t.plan.h, r(qrow), r(same), None) == 1
    for bad in ((-256, 64), (256, -64), (2 ** 41, 64)):
        assert L.mure_tokens_attend(t.cache.h, t.plan.h, r(rows(t.q.data_ptr(), *bad)), r(orow), None) == 1
    assert L.mure_tokens_attend(t.cache.h, t.plan.h, r(qrow), r(orow), out.data_ptr() + 2) == 1
    # another geometry's plan, another context's plan
    u = Batch(M, ctx, [2], [14], [16], 4, 2, 64, 8, "bf16", "same")
    assert L.mure_tokens_attend(t.cache.h, u.plan.h, r(qrow), r(orow), None) == 1
    other = M.mure_create(0)
    w = Batch(M, other, [2], [14], [16], 4, 2, 64, 16, "bf16", "same")
    assert L.mure_tokens_attend(t.cache.h, w.plan.h, r(qrow), r(orow), None) == 1
    # new tokens past the cells: they attend, but cannot be written or read
    p = M.mure_tokens_plan(t.cache, 4, [2], [15], [16], t.table)
    M.mure_tokens_attend(t.cache, p, t.q)
    for call in (lambda: M.mure_tokens_append(t.cache, p, t.k, t.v), lambda: M.mure_tokens_read(t.cache, p, new=True)):
        with pytest.raises(M.MureError) as ei:
            call()
        assert ei.value.status == 1
    for bad in (t.q.float(), t.q[:1], t.q.transpose(1, 2), t.q.cpu()):
        with pytest.raises(ValueError):
            M.mure_tokens_attend(t.cache, t.plan, bad)
    M.mure_synchronize(ctx)
    assert not bool(out.any()) and all(torch.equal(a, b) for a, b in zip(before, t.pools))
