"""Trees of new tokens on the GPU: attention over the earlier cells and the ancestors' against the 64-bit form, with the
tolerances of test_gpu_tokens.py; cells of kept paths, copied pages, and a run of all of it."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_tokens import M, TYPES, UNIT, Batch, ctx  # noqa: E402,F401


def grow(n, branch, rng, roots=0.1):
    """Parents of n tokens: one of the `branch` before, now and then none."""
    return [-1 if i == 0 or rng.random() < roots else int(rng.integers(max(0, i - branch), i)) for i in range(n)]


class Tree(Batch):
    """Batch, its new tokens trees.

    Beside test_gpu_tokens.py's tolerances, f16: a probability is held as an f16 number P = 2^(s - m), m at least 7 below the
    row's largest score, so that the largest P is 2^7 or more and one below f16's normal numbers is off by
    2^-25, half their least step: by 2^-25 / 2^7 = 2^-32 of the row's sum or less.  Over all cells that is
    2^-32 sum |v|.  Cells of codes are f16 numbers for the products: half a least step, 2^-25, off, as the output is."""

    def __init__(self, M, ctx, new, pos, kv, *a, parents=None, branch=4, **k):  # noqa: F811
        rng = np.random.default_rng(k.get("seed", 0))
        self.parents = parents or [grow(n, branch, rng) for n in new]
        super().__init__(M, ctx, new, pos, kv, *a, **k)

    def make_plan(self, plan=None):
        return self.M.mure_tokens_plan(self.cache, self.heads, self.new, self.pos, self.kv, self.table, window=self.window,
                                       sinks=self.sinks, scale=self.scale, plan=plan, parents=[p for x in self.parents for p in x])

    def depths(self, b):
        d = []
        for p in self.parents[b]:
            d.append(0 if p < 0 else d[p] + 1)
        return d

    def seen(self, b):
        n, pos, kv = self.new[b], self.pos[b], self.kv[b]
        depth = self.depths(b)
        see = np.zeros((n, max(kv, pos + n)), bool)
        at = np.arange(see.shape[1])
        at[pos:pos + n] = pos + np.array(depth, np.int64)
        for i in range(n):
            see[i, :pos] = True
            a = i
            while a >= 0:
                see[i, pos + a] = True
                a = self.parents[b][a]
            if self.window:
                see[i] &= (at > pos + depth[i] - self.window) | (at < self.sinks)
        return torch.from_numpy(see[:, :kv]).cuda()

    def reference(self):
        outs, lses, tols, ltols, row, grp = [], [], [], [], 0, self.heads // self.hk
        scale, u = self.scale or self.d ** -0.5, UNIT[self.dtype]
        for b, n in enumerate(self.new):
            if n == 0:
                continue
            k, v, see = self.dense(0, b), self.dense(1, b), self.seen(b)
            q = self.q[row:row + n].double()
            row += n
            out = torch.zeros(n, self.heads, self.d, dtype=torch.float64, device="cuda")
            lse = torch.full((n, self.heads), -math.inf, dtype=torch.float64, device="cuda")
            tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
            bad_v, bad_k = ~torch.isfinite(v), ~torch.isfinite(k).all(-1)
            kf, vf = k.nan_to_num(0, 0, 0), v.nan_to_num(0, 0, 0)
            for h in range(self.heads if self.kv[b] else 0):
                j = h // grp
                s = (q[:, h] @ kf[:, j].T * scale).masked_fill(~see, -math.inf)
                s = torch.where(see & bad_k[None, :, j], torch.full_like(s, math.nan), s)
                lse[:, h] = torch.logsumexp(s, -1)
                p = torch.where(see, torch.exp(s - lse[:, h:h + 1]), torch.zeros_like(s))
                A = p @ vf[:, j].abs()
                out[:, h] = (p @ vf[:, j]).masked_fill(see.double() @ bad_v[:, j].double() > 0, math.nan)
                E = torch.where(see, q[:, h].abs() @ kf[:, j].abs().T * scale, torch.zeros_like(s)).amax(-1)
                c = 2.0 ** -24 * (8 * math.sqrt(self.d) * E + 8 * math.sqrt(self.kv[b]) + 64)
                tol[:, h] = u * out[:, h].abs() + (u + c[:, None]) * A + 1e-30
                if self.dtype == "f16":
                    tol[:, h] += 2.0 ** -32 * (see.double() @ vf[:, j].abs()) + 2.0 ** -24
                ltol[:, h] = c * (1 + lse[:, h].abs())
            empty = ~see.any(-1)
            out[empty], lse[empty], tol[empty] = 0.0, -math.inf, 0.0
            outs.append(out); lses.append(lse); tols.append(tol); ltols.append(ltol)
        return torch.cat(outs), torch.cat(tols), torch.cat(lses), torch.cat(ltols)


# -------------------------------------------------------------- attention --

@pytest.mark.parametrize("form", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("heads,hk,d,page", [(8, 2, 128, 16), (4, 4, 64, 64), (15, 3, 40, 8), (2, 1, 256, 32), (16, 2, 96, 128)])
def test_trees(M, ctx, dtype, form, heads, hk, d, page):  # noqa: F811
    """Few rows and many, trees that start anywhere in a tile or a word, before any earlier cell and after many."""
    new, pos = [1, 0, 5, 33, 64, 65, 130], [0, 9, 700, 31, 1000, 0, 257]
    t = Tree(M, ctx, new, pos, [a + b for a, b in zip(new, pos)], heads, hk, d, page, dtype, form, seed=d)
    first = [x.clone() for x in t.check()]
    again = t.check()
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("form", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 0), (3, 50), (16, 4), (100, 700), (500, 1)])
def test_windows(M, ctx, dtype, form, window, sinks):  # noqa: F811
    """The window goes by positions: a token's ancestors further up than that are hidden, its siblings' cells lie
    between.  Sinks that end before, inside and after the tree."""
    new, pos = [20, 60, 7, 1], [650, 40, 3000, 0]
    t = Tree(M, ctx, new, pos, [a + b for a, b in zip(new, pos)], 6, 2, 64, 16, dtype, form, window=window, sinks=sinks, branch=2)
    t.check()


@pytest.mark.parametrize("branch,roots", [(1, 0.0), (1000, 0.0), (3, 0.0), (1, 1.0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shapes_of_trees(M, ctx, dtype, branch, roots):  # noqa: F811
    """A chain, a bush, a tree of little branching, and tokens without ancestors; up to the most tokens of a tree."""
    rng = np.random.default_rng(5)
    new = [1024, 300, 31, 32]
    pos = [77, 0, 1, 2000]
    t = Tree(M, ctx, new, pos, [a + b for a, b in zip(new, pos)], 2, 1, 64, 16, dtype, "same",
             parents=[grow(n, branch, rng, roots) for n in new])
    out, lse = t.check()
    if branch == 1 and roots == 0:               # a chain is an ordinary batch
        plan = M.mure_tokens_plan(t.cache, t.heads, t.new, t.pos, t.kv, t.table)
        t.check(M.mure_tokens_attend(t.cache, plan, t.q, lse=True))


@pytest.mark.parametrize("dtype,form", [("bf16", "same"), ("f16", "e4m3"), ("f32", "same")])
def test_trees_past_the_cells_held(M, ctx, dtype, form):  # noqa: F811
    """Cells that end inside the tree, before it, or that are not there: rows without any give zeros."""
    new, pos, kv = [40, 100, 9, 200], [100, 50, 30, 10], [113, 50, 0, 4]
    t = Tree(M, ctx, new, pos, kv, 4, 2, 64, 16, dtype, form, window=12)
    out, lse = t.check()
    assert not bool(out[140:149].any()) and bool((lse[140:149] == -math.inf).all())
    t = Tree(M, ctx, new, pos, kv, 4, 2, 64, 16, dtype, form)
    t.check()


@pytest.mark.parametrize("dtype,form", [("bf16", "same"), ("f16", "same"), ("f32", "same"), ("bf16", "e4m3"), ("f16", "e4m3"), ("f32", "e4m3")])
@pytest.mark.parametrize("new", [6, 90])
def test_masked_cells_may_hold_anything(M, ctx, dtype, form, new):  # noqa: F811
    """NaN and infinities in the cells of one branch reach its own tokens alone."""
    parents = [[-1, 0, 0] + [1 if i % 2 else 2 for i in range(new - 3)]]
    t = Tree(M, ctx, [new], [300], [300 + new], 8, 2, 64, 16, dtype, form, parents=parents)
    clean = t.check()[0].clone()
    at = (int(t.table[0, 301 // 16]), slice(None), 301 % 16)            # token 1's cell
    if form == "e4m3":
        t.pools[2][at] = 255
        t.pools[3][at] = 255
    else:
        t.pools[0][at] = math.nan
        t.pools[1][at] = math.inf if dtype != "bf16" else math.nan
    got = t.M.mure_tokens_attend(t.cache, t.plan, t.q, lse=True)
    M.mure_synchronize(ctx)
    hit = [i for i in range(new) if i == 1 or parents[0][i] == 1]
    free = [i for i in range(new) if i not in hit]
    assert bool(torch.isnan(got[0][hit]).all())
    assert bool(torch.isfinite(got[0][free]).all())
    ref, tol, _, _ = t.reference()
    assert bool(((got[0].double() - ref).abs() <= tol)[free].all())
    assert bool(((got[0].double() - clean.double()).abs() <= 2 * tol)[free].all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [128, 64, 96, 40, 16])
def test_codes_of_all_scales(M, ctx, dtype, d):  # noqa: F811
    """Scale bytes from the least to far past the common ones, NaN codes in masked cells and in one that some rows see: trees
    of many rows widen codes by short cuts that have to give the definition's values."""
    t = Tree(M, ctx, [90, 70], [700, 130], [790, 200], 8, 2, d, 16, dtype, "e4m3", seed=d, branch=6)
    g = torch.Generator(device="cuda").manual_seed(1)
    for which, (lo, hi) in ((2, (100, 128)), (3, (96, 134) if dtype == "f16" else (96, 150))):
        t.pools[which].copy_(torch.randint(lo, hi, t.pools[which].shape, generator=g, device="cuda").to(torch.uint8))
    t.pools[3][:, :, ::5] = 0
    t.pools[2][:, :, 1::7] = 0
    t.pools[2][:, :, 2::7] = 111
    t.pools[2][:, :, 3::7] = 112
    t.check()
    cell = 40                                              # of sequence 0's tree: its own row and its descendants'
    at = (int(t.table[0, (700 + cell) // 16]), slice(None), (700 + cell) % 16)
    t.pools[1].view(torch.uint8)[at][:, d // 2] = 0x7F
    t.pools[0].view(torch.uint8)[(int(t.table[1, 3]), slice(None), 5)][:, 1] = 0xFF
    out, _ = M.mure_tokens_attend(t.cache, t.plan, t.q, lse=True)
    M.mure_synchronize(ctx)
    hit = t.seen(0)[:, 700 + cell]
    assert bool(torch.isnan(out[:90][hit][..., d // 2]).all()) and bool(torch.isfinite(out[:90][~hit]).all())
    assert bool(torch.isnan(out[90:]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [128, 64])
def test_shared_pages_of_codes(M, ctx, dtype, d):  # noqa: F811
    """Trees over one sequence's pages (which are then widened once) give the bits that they give over pages of their
    own (which each piece widens)."""
    n, new, past, pages = 4, 60, 1000, -(-1060 // 16)
    own = Tree(M, ctx, [new] * n, [past] * n, [past + new] * n, 8, 2, d, 16, dtype, "e4m3", parents=[grow(new, 5, np.random.default_rng(2))] * n)
    for p in own.pools:                                     # all sequences' cells are sequence 0's
        p = p.view(torch.uint8)
        first = torch.from_numpy(own.table[0, :pages].astype(np.int64)).cuda()
        for b in range(1, n):
            p[torch.from_numpy(own.table[b, :pages].astype(np.int64)).cuda()] = p[first]
    apart = own.check()
    plan = M.mure_tokens_plan(own.cache, 8, own.new, own.pos, own.kv, np.repeat(own.table[:1], n, 0), parents=[p for x in own.parents for p in x])
    shared = M.mure_tokens_attend(own.cache, plan, own.q, lse=True)
    M.mure_synchronize(ctx)
    assert torch.equal(apart[0], shared[0]) and torch.equal(apart[1], shared[1])


def test_expired_waits(M):
    """Trees whose waits run out at once give TIMEOUT, and the same plans work again after it."""
    ctx = M.mure_create(0)  # noqa: F811
    trees = [Tree(M, ctx, [60, 20], [900, 300], [960, 320], heads, 2, 128, 16, "bf16", form)
             for heads, form in ((8, "same"), (4, "same"), (8, "e4m3"))]
    for t in trees:
        t.check()
    for t in trees:
        M.mure_set_wait_limit(ctx, 1)
        M.mure_tokens_attend(t.cache, t.plan, t.q)
        with pytest.raises(M.MureError) as ei:
            M.mure_synchronize(ctx)
        assert ei.value.status == 5
        M.mure_set_wait_limit(ctx, 0)
        t.check()


def test_long_pasts(M, ctx):  # noqa: F811
    """Trees over a long axis, split and joined, in every form."""
    for dtype, form in (("bf16", "same"), ("f16", "e4m3"), ("f32", "same"), ("bf16", "e4m3")):
        Tree(M, ctx, [3, 70], [40001, 20000], [40004, 20070], 4, 1, 64, 64, dtype, form).check()


def test_plans_change_between_trees_and_chains(M, ctx):  # noqa: F811
    t = Tree(M, ctx, [30, 4], [100, 90], [130, 94], 4, 2, 64, 16, "bf16", "same")
    first = t.check()[0].clone()
    M.mure_tokens_plan(t.cache, 4, t.new, t.pos, t.kv, t.table, plan=t.plan)
    chain = Batch.reference(t)
    got = M.mure_tokens_attend(t.cache, t.plan, t.q)
    M.mure_synchronize(ctx)
    assert bool(((got.double() - chain[0]).abs() <= chain[1]).all())
    t.make_plan(t.plan)
    assert torch.equal(t.check()[0], first)


def test_rotation_goes_by_depth(M, ctx):  # noqa: F811
    """Without positions of its own, a tree's token is rotated by its depth."""
    t = Tree(M, ctx, [9, 0, 33], [100, 5, 2], [109, 5, 35], 4, 2, 64, 16, "f32", "same")
    r = M.mure_rotary_create(ctx, 64)
    at = torch.tensor([p + d for b, p in enumerate(t.pos) for d in t.depths(b)], dtype=torch.int32, device="cuda")
    a, b = M.mure_tokens_rotate(t.cache, t.plan, r, t.q, t.k), M.mure_tokens_rotate(t.cache, t.plan, r, t.q, t.k, positions=at)
    M.mure_synchronize(ctx)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------ kept tokens --

def raw(t, which, b, j):
    """Bits of cell j of sequence b."""
    return t.pools[which].view(torch.uint8)[int(t.table[b, j // t.page]), :, j % t.page]


@pytest.mark.parametrize("dtype,form", [("bf16", "same"), ("f16", "e4m3"), ("f32", "same"), ("f32", "e4m3")])
@pytest.mark.parametrize("hk,d,page", [(2, 64, 16), (5, 40, 8), (1, 256, 64), (40, 128, 8), (3, 8, 1024)])
def test_keep(M, ctx, dtype, form, hk, d, page):  # noqa: F811
    """Paths of every kind move up, bit for bit; no other cell changes."""
    rng = np.random.default_rng(d)
    new, pos = [40, 0, 1, 100, 17, 64], [3, 5, 0, 2 * page - 1, 100, 30]
    t = Tree(M, ctx, new, pos, [a + b + 2 for a, b in zip(new, pos)], hk, hk, d, page, dtype, form)
    kept = [sorted(rng.choice(n, rng.integers(0, n + 1), replace=False).tolist()) if n else [] for n in new]
    kept[3] = list(range(60)) + [99]             # most of it stays where it is
    kept[5] = list(range(32, 64))                # all of it by half
    before = [p.clone() for p in t.pools]
    M.mure_tokens_keep(t.cache, t.plan, kept)
    M.mure_synchronize(ctx)
    for w in range(len(t.pools)):
        want = before[w].view(torch.uint8).clone()
        for b, path in enumerate(kept):
            for to, i in enumerate(path):
                src, dst = pos[b] + i, pos[b] + to
                want[int(t.table[b, dst // page]), :, dst % page] = before[w].view(torch.uint8)[int(t.table[b, src // page]), :, src % page]
        assert torch.equal(t.pools[w].view(torch.uint8), want)


def test_keep_of_many(M, ctx):  # noqa: F811
    """More sequences and more kept tokens than one launch takes, an ordinary chunk's among them."""
    n = 700
    new = [2] * n + [15000]
    pos = [3] * n + [1]
    t = Batch(M, ctx, new, pos, [a + b for a, b in zip(new, pos)], 1, 1, 8, 16, "bf16", "same")
    kept = [[1]] * n + [list(range(1, 15000))]
    before = t.pools[0].clone()
    launches = M.mure_kernel_launches(ctx)
    M.mure_tokens_keep(t.cache, t.plan, kept)
    assert M.mure_kernel_launches(ctx) - launches > 2
    M.mure_synchronize(ctx)
    old, now = before[t.table[n, :].astype(np.int64)].transpose(1, 2).reshape(-1, 8), t.pools[0][t.table[n].astype(np.int64)].transpose(1, 2).reshape(-1, 8)
    assert torch.equal(now[1:15000], old[2:15001]) and torch.equal(now[0], old[0]) and torch.equal(now[15000:], old[15000:])
    ids = torch.from_numpy(t.table[:n, 0].astype(np.int64)).cuda()
    assert torch.equal(t.pools[0][ids, :, 3], before[ids, :, 4]) and torch.equal(t.pools[0][ids, :, 4], before[ids, :, 4])


# ----------------------------------------------------------- copied pages --

@pytest.mark.parametrize("dtype,form", [("bf16", "same"), ("f16", "e4m3"), ("f32", "same")])
@pytest.mark.parametrize("hk,d,page,n", [(2, 64, 16, 1), (5, 40, 8, 64), (3, 8, 8, 65), (1, 256, 1024, 3), (1, 8, 8, 4001), (8, 128, 16, 300)])
def test_copy_pages(M, ctx, dtype, form, hk, d, page, n):  # noqa: F811
    """Pages of the cache itself and of another one, one source for several targets; no other page changes."""
    t = Batch(M, ctx, [0], [0], [0], hk, hk, d, page, dtype, form, spare=2 * n + 5)
    u = Batch(M, ctx, [0], [0], [0], hk, hk, d, page, dtype, form, spare=n + 2, seed=1)
    order = np.random.default_rng(n).permutation(t.n_pages)
    src, dst = order[:n].copy(), order[n:2 * n]
    src[: n // 2] = src[0]
    before = [p.clone() for p in t.pools]
    M.mure_tokens_copy_pages(t.cache, src, dst)
    M.mure_synchronize(ctx)
    a, b = (torch.from_numpy(x.astype(np.int64)).cuda() for x in (src, dst))
    for p, q in zip(t.pools, before):
        q.view(torch.uint8)[b] = q.view(torch.uint8)[a]
        assert torch.equal(p.view(torch.uint8), q.view(torch.uint8))
    far = np.arange(n)[::-1]
    kept = [p.clone() for p in t.pools]
    M.mure_tokens_copy_pages(u.cache, src, far, source=t.cache)
    M.mure_synchronize(ctx)
    for p, q in zip(u.pools, t.pools):
        assert torch.equal(p.view(torch.uint8)[torch.from_numpy(far.copy()).cuda()], q.view(torch.uint8)[a])
    assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(kept, t.pools))


# -------------------------------------------------------------- refusals --

def test_tree_refusals(M, ctx):  # noqa: F811
    import ctypes as C
    t = Batch(M, ctx, [3], [13], [16], 4, 2, 64, 16, "bf16", "same")

    def plan(parents, new=(3,), pos=(13,), **k):
        return M.mure_tokens_plan(t.cache, 4, list(new), list(pos), [16] * len(new), np.zeros((len(new), 1), np.int32), parents=parents, **k)

    p = plan([-1, 0, 0])
    for bad in ([0, 0, 0], [-1, 1, 0], [-1, 0, 2], [-2, 0, 0], [-1, 0, 5], [-1, 0, -2 ** 31]):
        with pytest.raises(M.MureError) as ei:
            plan(bad)
        assert ei.value.status == 1, bad
    with pytest.raises(M.MureError) as ei:                 # parents are a sequence's own
        plan([-1, 0, -1, 2, 3, 4], new=(2, 4), pos=(0, 0))
    assert ei.value.status == 1
    for bad in ([-1, 0], [-1, 0, 0, 0], [], [0.5, 0, 0], [2 ** 32 - 1, 0, 0]):
        with pytest.raises(ValueError):
            plan(bad)
    with pytest.raises(M.MureError) as ei:
        plan([-1] * 1025, new=(1025,), pos=(0,))
    assert ei.value.status == 2
    b, _keep = M._tokens_batch(4, [3], [13], [16], np.zeros((1, 1), np.int32), 0, 0, 0.0)
    out = C.c_void_p(7)
    assert M.lib().mure_tokens_plan_create_tree(t.cache.h, C.byref(b), None, C.byref(out)) == 1 and not out.value
    assert M.lib().mure_tokens_plan_set_tree(p.h, C.byref(b), None) == 1
    with pytest.raises(M.MureError):                       # ... and the plan now holds none
        M.mure_tokens_attend(t.cache, p, t.q)
    plan([], new=(0,), pos=(0,))
    plan([], new=(), pos=())


def test_keep_refusals(M, ctx):  # noqa: F811
    t = Batch(M, ctx, [3, 2], [13, 0], [16, 2], 4, 2, 64, 16, "bf16", "same")
    before = [p.clone() for p in t.pools]
    for bad in ([[0, 1, 2, 2], []], [[1, 0], []], [[0, 0], []], [[3], []], [[-1], []], [[], [2]], [[0], [1, 1]]):
        with pytest.raises(M.MureError) as ei:
            M.mure_tokens_keep(t.cache, t.plan, bad)
        assert ei.value.status == 1, bad
    for bad in ([[0]], [[0], [0], [0]], [[0.5], []], [[2 ** 32], []]):
        with pytest.raises(ValueError):
            M.mure_tokens_keep(t.cache, t.plan, bad)
    count = np.array([1, 0], np.int32)
    L = M.lib()
    assert L.mure_tokens_keep(t.cache.h, t.plan.h, None, None) == 1
    assert L.mure_tokens_keep(t.cache.h, t.plan.h, count.ctypes.data, None) == 1
    assert L.mure_tokens_keep(t.cache.h, None, count.ctypes.data, count.ctypes.data) == 1
    count[0] = -1
    assert L.mure_tokens_keep(t.cache.h, t.plan.h, count.ctypes.data, count.ctypes.data) == 1
    M.mure_tokens_keep(t.cache, t.plan, [[], []])
    M.mure_tokens_keep(t.cache, t.plan, [[0, 1, 2], [0]])
    p = M.mure_tokens_plan(t.cache, 4, [2], [15], [16], t.table)              # past the cells
    with pytest.raises(M.MureError):
        M.mure_tokens_keep(t.cache, p, [[1]])
    p = M.mure_tokens_plan(t.cache, 4, [2, 2], [5, 5], [7, 7], np.zeros((2, 1), np.int32))
    with pytest.raises(M.MureError):                                          # two sequences' cells are the same
        M.mure_tokens_keep(t.cache, p, [[1], [1]])
    M.mure_synchronize(ctx)
    assert all(torch.equal(a, b) for a, b in zip(before, t.pools))


def test_copy_refusals(M, ctx):  # noqa: F811
    t = Batch(M, ctx, [0], [0], [0], 2, 2, 64, 16, "bf16", "same", spare=8)
    before = [p.clone() for p in t.pools]
    for src, dst in (([0], [8]), ([8], [0]), ([-1], [0]), ([0], [-1]), ([0, 1], [5, 5]), ([0, 5], [5, 6]), ([3], [3]), (range(9), range(9))):
        with pytest.raises(M.MureError) as ei:
            M.mure_tokens_copy_pages(t.cache, list(src), list(dst))
        assert ei.value.status == 1, (src, dst)
    for src, dst in (([0], [1, 2]), ([0.5], [1]), ([2 ** 32], [1])):
        with pytest.raises(ValueError):
            M.mure_tokens_copy_pages(t.cache, src, dst)
    M.mure_tokens_copy_pages(t.cache, [], [])
    other = Batch(M, ctx, [0], [0], [0], 2, 2, 64, 8, "bf16", "same", spare=8)
    away = Batch(M, M.mure_create(0), [0], [0], [0], 2, 2, 64, 16, "bf16", "same", spare=8)
    # a second handle on the same pools, and one on a part of them
    twin = M.mure_tokens_create(ctx, 2, 64, 16, 8, dtype="bf16", buffers=tuple(t.pools))
    part = M.mure_tokens_create(ctx, 2, 64, 16, 6, dtype="bf16", buffers=tuple(p[2:] for p in t.pools))
    for source in (other.cache, away.cache, part):
        with pytest.raises(M.MureError) as ei:
            M.mure_tokens_copy_pages(t.cache, [0], [1], source=source)
        assert ei.value.status == 1
    with pytest.raises(M.MureError):
        M.mure_tokens_copy_pages(t.cache, [0, 1], [1, 2], source=twin)
    L = M.lib()
    ids = np.array([0], np.int32)
    assert L.mure_tokens_copy_pages(t.cache.h, t.cache.h, -1, ids.ctypes.data, ids.ctypes.data) == 1
    assert L.mure_tokens_copy_pages(t.cache.h, t.cache.h, 1, None, ids.ctypes.data) == 1
    assert L.mure_tokens_copy_pages(t.cache.h, None, 1, ids.ctypes.data, ids.ctypes.data) == 1
    M.mure_synchronize(ctx)
    assert all(torch.equal(a, b) for a, b in zip(before, t.pools))
    M.mure_tokens_copy_pages(t.cache, [0], [1], source=twin)
    M.mure_synchronize(ctx)
    assert torch.equal(t.pools[0][1], before[0][0])


# ------------------------------------------------------------- a run of it --

@pytest.mark.parametrize("dtype,form", [("bf16", "same"), ("f16", "e4m3"), ("f32", "same")])
def test_steps(M, ctx, dtype, form):  # noqa: F811
    """Three steps of two sequences: rotated and stored as a tree, attended, a path kept; then one of them is forked and
    both continue.  The cells are, bit for bit, those of the kept tokens stored one after the other, and the kept
    path's last token attends as an ordinary one."""
    heads, hk, d, page, dt = 4, 2, 64, 16, TYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(3)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    tree = M.mure_tokens_create(ctx, hk, d, page, 64, dtype=dtype, form=form)
    line = M.mure_tokens_create(ctx, hk, d, page, 64, dtype=dtype, form=form)
    w = np.linspace(0.5, 1.5, d).astype(np.float32)
    rot = M.mure_rotary_create(ctx, d, 48, q_weight=w, k_weight=w[::-1].copy())
    table = np.arange(40, dtype=np.int32).reshape(2, 20)
    rng = np.random.default_rng(0)
    held = [0, 0]
    for step in range(4):
        if step == 3:                                      # sequence 1 becomes a fork of sequence 0
            full = held[0] // page
            table[1, :full] = table[0, :full]
            if held[0] % page:
                for c in (tree, line):
                    M.mure_tokens_copy_pages(c, [int(table[0, full])], [60])
                table[1, full] = 60
            held[1] = held[0]
        new = [int(rng.integers(3, 40)), int(rng.integers(1, 20))]
        parents = [grow(n, 3, rng, 0.0) for n in new]
        kept = []
        for p in parents:
            path, i = [], len(p) - 1
            while i >= 0:
                path.append(i)
                i = p[i]
            kept.append(path[::-1])
        n = sum(new)
        q, k, v = make(n, heads, d), make(n, hk, d), make(n, hk, d)
        plan = M.mure_tokens_plan(tree, heads, new, held, [a + b for a, b in zip(held, new)], table, parents=[i for p in parents for i in p])
        out, lse = M.mure_tokens_attend(tree, plan, M.mure_tokens_append_rotated(tree, plan, rot, q, k, v), lse=True)
        M.mure_tokens_keep(tree, plan, kept)
        rows = torch.tensor([i + new[0] * b for b, path in enumerate(kept) for i in path], device="cuda")
        m = [len(path) for path in kept]
        flat = M.mure_tokens_plan(line, heads, m, held, [a + b for a, b in zip(held, m)], table)
        qr = M.mure_tokens_append_rotated(line, flat, rot, q[rows].contiguous(), k[rows].contiguous(), v[rows].contiguous())
        want, wlse = M.mure_tokens_attend(line, flat, qr, lse=True)
        M.mure_synchronize(ctx)
        # two computations of one value: within twice the rounding and the probabilities' (16 bits)
        u = UNIT[dtype]
        tol = 4 * u * (v.float().abs().max().double() + 1) + 2.0 ** -24 * 1e4
        assert float((out[rows].double() - want.double()).abs().max()) <= tol
        assert float((lse[rows] - wlse).abs().max()) <= 2.0 ** -24 * 1e4
        held = [a + b for a, b in zip(held, m)]
        dense = [M.mure_tokens_read(c, M.mure_tokens_plan(c, heads, [0, 0], [0, 0], held, table)) for c in (tree, line)]
        for a, b in zip(*dense):
            assert torch.equal(a, b)
    M.mure_synchronize(ctx)


def test_captured_steps(M):
    """Two steps captured in graphs, on a context of its own stream, replayed in turn with other inputs: each gives what
    the calls give."""
    s = torch.cuda.Stream()
    ctx = M.mure_create(0, stream=s)  # noqa: F811
    runs = []
    with torch.cuda.stream(s):
        for seed, form in ((0, "same"), (1, "e4m3")):
            t = Tree(M, ctx, [40, 3, 17], [100, 64, 0], [140, 67, 17], 8, 2, 64, 16, "bf16", form, seed=seed)
            r = M.mure_rotary_create(ctx, 64, q_weight=np.ones(64, np.float32), k_weight=np.ones(64, np.float32))
            kept = [[0, 5, 20, 39], [1], [0, 16]]

            def step(t=t, r=r, kept=kept):
                q = M.mure_tokens_append_rotated(t.cache, t.plan, r, t.q, t.k, t.v)
                out = M.mure_tokens_attend(t.cache, t.plan, q, lse=True)
                M.mure_tokens_keep(t.cache, t.plan, kept)
                M.mure_tokens_copy_pages(t.cache, [int(t.table[0, 0])], [t.n_pages - 1] if t.n_pages - 1 not in t.table else [int(t.table[1, 0])])
                return out
            step()
            M.mure_synchronize(ctx)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                out = step()
            runs.append((t, step, graph, out))
        for turn in range(3):
            for t, step, graph, out in runs:
                for x in (t.q, t.k, t.v):
                    x.copy_(torch.randn(x.shape, device="cuda"))
                pools = [p.clone() for p in t.pools]
                graph.replay()
                got = [x.clone() for x in out] + [p.clone() for p in t.pools]
                for p, q in zip(t.pools, pools):
                    p.copy_(q)
                want = list(step()) + t.pools
                M.mure_synchronize(ctx)
                for a, b in zip(got, want):
                    assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_captured_joins(M):
    """Trees whose rows are split and joined, captured: replays give the calls' bits, also behind other work."""
    s = torch.cuda.Stream()
    ctx = M.mure_create(0, stream=s)  # noqa: F811
    with torch.cuda.stream(s):
        for heads, form in ((4, "same"), (16, "same"), (16, "e4m3")):
            t = Tree(M, ctx, [30, 12], [6000, 3000], [6030, 3012], heads, 2, 128, 16, "bf16", form)
            before = M.mure_kernel_launches(ctx)
            want = [x.clone() for x in M.mure_tokens_attend(t.cache, t.plan, t.q, lse=True)]
            assert M.mure_kernel_launches(ctx) - before >= 2
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                x = torch.zeros(1 << 22, device="cuda")
                x += 1
                got = M.mure_tokens_attend(t.cache, t.plan, t.q, lse=True)
                y = got[0].clone()
            for _ in range(20):
                for g in got:
                    g.fill_(7)
                graph.replay()
                assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(y, want[0])
            M.mure_synchronize(ctx)


def test_another_stream(M):
    """A context on a stream of its own, called from torch's current one."""
    ctx = M.mure_create(0, stream=torch.cuda.Stream())  # noqa: F811
    t = Tree(M, ctx, [30], [50], [80], 4, 2, 64, 16, "bf16", "same")
    r = M.mure_rotary_create(ctx, 64)
    for i in range(20):
        x = torch.full((30, 2, 64), float(i + 1), device="cuda", dtype=torch.bfloat16)
        q = torch.full((30, 4, 64), 1.0, device="cuda", dtype=torch.bfloat16)
        got, _ = M.mure_tokens_rotate(t.cache, t.plan, r, q)
        M.mure_tokens_append_rotated(t.cache, t.plan, r, None, x, x)
        M.mure_tokens_keep(t.cache, t.plan, [[29]])
        M.mure_tokens_copy_pages(t.cache, [int(t.table[0, 3])], [t.n_pages - 1] if t.n_pages - 1 not in t.table[0] else [int(t.table[0, 0])])
        del x, q
        torch.full((30, 4, 64), -5.0, device="cuda", dtype=torch.bfloat16)
        _, v = M.mure_tokens_read(t.cache, t.plan, new=True)
        assert bool((v == i + 1).all()) and bool((got.float().abs() <= 1.5).all())
    M.mure_synchronize(ctx)
