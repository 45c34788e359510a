"""Token caches where calls go wrong first: work without cells beside work with some, scales and values at the
ends of their range, long sums, rows computed again by the definition, arguments that do not fit.  Attention
against the 64-bit form of test_gpu_tokens.py, with its tolerances."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_tokens import M, Batch, ctx  # noqa: E402,F401


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,pos", [(0, 0), (32, 900)])
def test_chunks_without_cells_after_short_ones(M, ctx, d, window, pos):  # noqa: F811
    """Blocks that go from one short piece with cells to several of twice the rows without any (no cells held,
    or a window past them): zeros there, no wait that runs out."""
    new = [128] * 200 + [256] * 300
    at = [70] * 200 + [pos] * 300
    kv = [198] * 200 + [0 if window == 0 else 60] * 300
    t = Batch(M, ctx, new, at, kv, 2, 2, d, 16, "bf16", "same", window=window)
    for _ in range(2):
        out, lse = t.check()
        assert not bool(out[200 * 128:].any()) and bool((lse[200 * 128:] == -math.inf).all())


def byte_at(t, b, j):
    """Index of cell j of sequence b in a pool, all heads."""
    return int(t.table[b, j // t.page]), slice(None), j % t.page


def compare(t, rows, got=None):
    """The given rows against 64 bits, with no allowance for an output below the tolerance's floor."""
    out, lse = got if got is not None else t.M.mure_tokens_attend(t.cache, t.plan, t.q, lse=True)
    t.M.mure_synchronize(t.ctx)
    ref, tol, rlse, ltol = (x[rows] for x in t.reference())
    assert bool(((out[rows].double() - ref).abs() <= tol).all()), float(((out[rows].double() - ref).abs() / tol).max())
    assert bool(((lse[rows].double() - rlse).abs() <= ltol).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,new", [(2, 2), (2, 8), (32, 2), (2, 100)])
@pytest.mark.parametrize("above", [24, 40, 48, 130])
def test_loud_values_in_masked_cells(M, ctx, dtype, heads, new, above):  # noqa: F811
    """A finite value 2^24 to 2^130 above all others in a cell that only a chunk's first token sees (the last
    cell before its window's end; the next token's own window starts after it), and one in the last token's own
    cell: the other rows' outputs are as if these cells were empty."""
    t = Batch(M, ctx, [new], [300], [300 + new], heads, 2, 64, 16, dtype, "e4m3", window=16)
    t.pools[3].copy_((t.pools[3].int() - 8 * (above > 100)).to(torch.uint8))
    for j in (300 - 15, 300 + new - 1):
        at = byte_at(t, 0, j)
        t.pools[3][at] = int(min(250, int(t.pools[3][byte_at(t, 0, 290)][0]) + above))
        t.pools[1].view(torch.uint8)[at] = 0x30        # 1/2
    compare(t, slice(1, new - 1) if new > 2 else slice(0, 0))
    if new == 2:                                       # (one row between the two: without the later cell)
        t.pools[3][byte_at(t, 0, 300 + new - 1)] = t.pools[3][byte_at(t, 0, 290)]
        compare(t, slice(1, 2))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads", [2, 16])
@pytest.mark.parametrize("above", [24, 30, 44, 56])
def test_loud_values_of_no_probability(M, ctx, dtype, heads, above):  # noqa: F811
    """A single token's loud cell is visible, but its score lies 250 below the others': it adds nothing, and
    takes no bits from what the others add.  (The others within f16.)"""
    t = Batch(M, ctx, [1], [500], [501], heads, 2, 64, 16, dtype, "e4m3", scale=1.0)
    t.q.fill_(1.0)
    t.pools[0].view(torch.uint8)[:] = 0
    t.pools[3].fill_(112 if dtype == "f16" else 100)   # values around 2^-8, 2^-20
    at = byte_at(t, 0, 123)
    t.pools[2][at] = 127
    t.pools[0].view(torch.uint8)[at] = 0xC8            # -4: a score of -256
    t.pools[3][at] = int(t.pools[3][0, 0, 0]) + above
    t.check()
    t.pools[3].clamp_(max=int(t.pools[3][at][0]) - above)
    t.check()


@pytest.mark.parametrize("loud", [10, 25, 60])
def test_least_scales_beside_larger_ones(M, ctx, loud):  # noqa: F811
    """Cells of the least scale byte with codes that are not zero, beside a masked cell of a larger scale: bf16 rows
    keep them.  (Their values, some 2^-119, lie below the tolerance's floor: compared times 2^60.)"""
    t = Batch(M, ctx, [2], [40], [42], 2, 2, 64, 16, "bf16", "e4m3", window=16)
    t.pools[3].fill_(0)
    t.pools[1].view(torch.uint8)[:] |= 0x70            # magnitudes 128 to 448
    t.pools[1].view(torch.uint8)[(t.pools[1].view(torch.uint8) & 0x7F) == 0x7F] -= 1
    t.pools[3][byte_at(t, 0, 41)] = loud               # the second token's own
    out, _ = M.mure_tokens_attend(t.cache, t.plan, t.q, lse=True)
    M.mure_synchronize(ctx)
    scaled = out.double() * 2.0 ** 60
    t.pools[3][t.pools[3] == 0] = 60
    ref, tol, _, _ = t.reference()
    assert bool(((scaled - ref).abs() <= tol)[0].all()), float(((scaled - ref).abs() / tol)[0].max())
    zero = t.pools[1].view(torch.uint8)
    zero[:] = 0                                        # rows of zeros of any scale are zeros
    t.pools[3][t.pools[3] == 60] = 0
    t.check()


@pytest.mark.parametrize("dtype,heads", [("bf16", 2), ("bf16", 32), ("f16", 2), ("f32", 2)])
def test_scores_whose_factors_pass_the_range(M, ctx, dtype, heads):  # noqa: F811
    """Keys of 2^124 against a query or a scale so small that the scores are a few units, all negative: the product
    before its last factor is beyond fp32, the score is not."""
    t = Batch(M, ctx, [1, 3], [200, 90], [201, 93], heads, 2, 64, 16, dtype, "e4m3", scale=2.0 ** -124 if dtype == "f16" else 1.0)
    t.q.copy_(torch.rand_like(t.q.float()) + 1)
    if dtype != "f16":
        t.q.mul_(2.0 ** -64).mul_(2.0 ** -64)          # (in two steps: 2^-128 is subnormal)
    t.pools[0].view(torch.uint8)[:] = 0xB8             # -1
    t.pools[0].view(torch.uint8)[:, :, ::3] = 0xB4     # -3/4
    t.pools[2].fill_(251)
    t.check()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("form", ["same", "e4m3"])
def test_fp32_sums_over_long_axes(M, ctx, form, d):  # noqa: F811
    """fp32 rows over 300,000 cells whose values have one sign and nearly equal probabilities, in pieces of work
    that are not cut (a sequence per resident block and more, all on the same pages): rounding errors must not
    add up on one side."""
    n, many = 300_000, 500
    t = Batch(M, ctx, [1], [n - 1], [n], 1, 1, d, 64, "f32", form)
    t.q.mul_(0.01)
    if form == "same":
        t.pools[1].abs_().add_(0.5)
    else:
        t.pools[1].view(torch.uint8).bitwise_and_(0x7F)
    ref, tol, rlse, ltol = t.reference()
    plan = M.mure_tokens_plan(t.cache, 1, [1] * many, [n - 1] * many, [n] * many, np.repeat(t.table, many, 0))
    out, lse = M.mure_tokens_attend(t.cache, plan, t.q.repeat(many, 1, 1), lse=True)
    M.mure_synchronize(ctx)
    assert bool(((out.double() - ref).abs() <= tol).all()), float(((out.double() - ref).abs() / tol).max())
    assert bool(((lse.double() - rlse).abs() <= ltol).all())


@pytest.mark.parametrize("dtype,form", [("bf16", "same"), ("f16", "e4m3")])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_done_again_are_no_expired_wait(M, d, dtype, form):  # noqa: F811
    """NaN in dead cells of every sequence's last page: its rows are computed again by the definition, which takes
    milliseconds a piece.  With waits limited to 2,000,000 cycles (a millisecond; the kernel's own last some
    microseconds) the other roles must not give up meanwhile, whatever the pieces before and after."""
    ctx = M.mure_create(0)
    new, past = [130, 256, 300, 70] * 50, [1500, 2000, 900, 2200] * 50
    t = Batch(M, ctx, new, past, [a + b for a, b in zip(new, past)], 2, 2, d, 16, dtype, form)
    for b, k in enumerate(t.kv):
        if k % t.page and b % 3:
            page = int(t.table[b, k // t.page])
            if form == "e4m3":
                t.pools[3][page, :, k % t.page:] = 255
            else:
                t.pools[1][page, :, k % t.page:] = math.nan
    M.mure_set_wait_limit(ctx, 2_000_000)
    for _ in range(2):
        out, _ = t.check()
        assert bool(torch.isfinite(out).all())
    M.mure_set_wait_limit(ctx, 0)


@pytest.mark.parametrize("new", [1, 100])
def test_f16_codes_beyond_f16(M, ctx, new):  # noqa: F811
    """Pools of the caller's whose codes times scales pass f16's range: keys of 2^24 against small queries, of
    both signs, and values of 2^18 with small probabilities.  What comes out does not depend on the number of
    new tokens."""
    t = Batch(M, ctx, [new], [260], [260 + new], 4, 2, 64, 16, "f16", "e4m3", scale=2.0 ** -20)
    t.q.mul_(0.01)
    t.pools[2].fill_(127 + 18)                         # K around 2^24
    lowest = t.pools[0].view(torch.uint8)
    lowest[:] &= 0xBF                                  # (magnitudes below 2)
    page, heads, slot = byte_at(t, 0, 57)
    t.q[..., 0] = 4.0
    lowest[..., 0] = 0x38                              # +1
    lowest[page, heads, slot, 0] = 0xD0                # -8: a score lower by 9
    t.pools[3].fill_(112)
    t.pools[3][page, heads, slot] = 127 + 8
    out, _ = t.check()
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("new", [1, 20, 200])
def test_f16_subnormals_come_back(M, ctx, new):  # noqa: F811
    """Each token attends to its own cell alone (a window of one): the output is the cell, bit for bit, down to
    f16's smallest numbers."""
    t = Batch(M, ctx, [new], [33], [33 + new], 8, 2, 64, 16, "f16", "e4m3", window=1)
    g = torch.Generator(device="cuda").manual_seed(2)
    v = torch.randint(-16, 17, (new, 2, 64), generator=g, device="cuda").half() * 2.0 ** -24
    M.mure_tokens_append(t.cache, t.plan, t.k, v)
    out = M.mure_tokens_attend(t.cache, t.plan, t.q)
    _, got = M.mure_tokens_read(t.cache, t.plan, new=True)
    M.mure_synchronize(ctx)
    assert torch.equal(got, v) and torch.equal(out, v.repeat_interleave(4, 1))


def test_plans_do_not_wait_for_the_stream(M):  # noqa: F811
    """A new batch of some 600 KB of tables in an existing plan, behind a tenth of a second of work on the context's
    stream: the call returns while that work still runs, and its tables are right."""
    s = torch.cuda.Stream()
    own = M.mure_create(0, stream=s)
    n, kv, page = 100, 12000, 8
    t = Batch(M, own, [1] * n, [kv - 1] * n, [kv] * n, 2, 1, 64, page, "bf16", "same")
    x = torch.randn(8192, 8192, device="cuda", dtype=torch.bfloat16)
    t.make_plan(t.plan)
    done = torch.cuda.Event()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        x @ x
        for _ in range(200):
            x @ x
        done.record()
        t.make_plan(t.plan)
        waited = done.query()
        out, lse = M.mure_tokens_attend(t.cache, t.plan, t.q, lse=True)
    assert not waited
    t.check((out, lse))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_up_to_the_largest(M, ctx, dtype):  # noqa: F811
    """A factor of the scores that leaves fp32 once it is in powers of two is refused; up to there scores of 0 are 0."""
    t = Batch(M, ctx, [1, 100], [50, 20], [51, 120], 4, 2, 64, 16, dtype, "same")
    t.q.zero_()
    t.scale = 2e38
    t.make_plan(t.plan)
    t.check()
    for scale in (2.4e38, 3.4e38):
        t.scale = scale
        with pytest.raises(M.MureError) as ei:
            t.make_plan(t.plan)
        assert ei.value.status == 1


def test_rows_that_require_gradients_are_refused(M, ctx):  # noqa: F811
    """No call records a gradient; none drops one silently."""
    t = Batch(M, ctx, [3], [14], [17], 4, 2, 64, 16, "bf16", "same")
    q, k = t.q.clone().requires_grad_(), t.k.clone().requires_grad_()
    before = [p.clone() for p in t.pools]
    calls = [lambda: M.mure_tokens_attend(t.cache, t.plan, q), lambda: M.mure_tokens_append(t.cache, t.plan, k, t.v),
             lambda: M.mure_tokens_append(t.cache, t.plan, t.k, k), lambda: M.mure_tokens_read(t.cache, t.plan, new=True, out=(k, t.v))]
    for call in calls:
        with pytest.raises(ValueError):
            call()
    M.mure_synchronize(ctx)
    assert all(torch.equal(a, b) for a, b in zip(before, t.pools))
    want = M.mure_tokens_attend(t.cache, t.plan, t.q)
    assert torch.equal(M.mure_tokens_attend(t.cache, t.plan, q.detach()), want)
    with torch.no_grad():
        assert torch.equal(M.mure_tokens_attend(t.cache, t.plan, q), want)
