"""Trees on e4m3 cells on the GPU: which way their codes are widened, and that either gives the same.

A plan that has pages widened first makes one launch more for each call than one whose pieces widen codes themselves, where
the same units are cut (they are: of the same rows and tiles)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_token_trees import Tree, grow  # noqa: E402
from test_gpu_tokens import M, ctx  # noqa: E402,F401


class Far(Tree):
    """Tree, its values so far apart that what fp32 does not hold of a probability counts.

    Powers of two go below fp32's normal numbers as 0.  They are taken of a row's scores less m, where the largest score yet lies 7
    to 15 above m.  So a probability that goes as 0, or goes with a factor 2^(m - m') that is 0 where m moves to m' or parts
    of a row are joined, is below 2^-126 2^15 / 2^7 = 2^-118 of the row's largest one, and thus of its sum: 2^-118
    sum |v| over its cells beside the other tolerances."""

    def reference(self):
        out, tol, lse, ltol = super().reference()
        row, grp = 0, self.heads // self.hk
        for b, n in enumerate(self.new):
            v, see = self.dense(1, b).nan_to_num(0, 0, 0).abs(), self.seen(b).double()
            for h in range(self.heads):
                tol[row:row + n, h] += 2.0 ** -118 * (see @ v[:, h // grp])
            row += n
        return out, tol, lse, ltol


def launches(M, ctx, cache, plan, q):  # noqa: F811
    """(kernel launches, outputs) of a call."""
    before = M.mure_kernel_launches(ctx)
    out = M.mure_tokens_attend(cache, plan, q, lse=True)
    return M.mure_kernel_launches(ctx) - before, out


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [128, 64, 16])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 20)])
def test_both_ways_give_the_same_bits(M, ctx, dtype, d, window, sinks):  # noqa: F811
    """Trees over pages of their own widen codes in their pieces, trees over one sequence's pages have these widened
    once, and the outputs are equal bit for bit, also at scales that leave the short cuts and with NaNs that rows see."""
    n, new, past = 5, 60, 1000
    t = Tree(M, ctx, [new] * n, [past] * n, [past + new] * n, 8, 2, d, 16, dtype, "e4m3", parents=[grow(new, 5, np.random.default_rng(2))] * n,
             window=window, sinks=sinks)
    g = torch.Generator(device="cuda").manual_seed(d)
    for which in (2, 3):
        t.pools[which].copy_(torch.randint(95, 128, t.pools[which].shape, generator=g, device="cuda").to(torch.uint8))
    # (NaNs where one tree's branch, or all rows, see them)
    t.pools[0].view(torch.uint8)[int(t.table[0, (past + 30) // 16]), :, (past + 30) % 16, 3] = 0x7F
    t.pools[3][int(t.table[0, 1010 // 16]), 1, 1010 % 16] = 255
    t.pools[1].view(torch.uint8)[int(t.table[0, 900 // 16]), 0, 900 % 16, 5] = 0xFF
    for p in t.pools:                                       # all sequences' cells are sequence 0's
        p = p.view(torch.uint8)
        first = torch.from_numpy(t.table[0, :-(-(past + new) // 16)].astype(np.int64)).cuda()
        for b in range(1, n):
            p[torch.from_numpy(t.table[b, :len(first)].astype(np.int64)).cuda()] = p[first]
    shared = M.mure_tokens_plan(t.cache, 8, t.new, t.pos, t.kv, np.repeat(t.table[:1], n, 0), window=window, sinks=sinks,
                                parents=[p for x in t.parents for p in x])
    a, apart = launches(M, ctx, t.cache, t.plan, t.q)
    b, once = launches(M, ctx, t.cache, shared, t.q)
    M.mure_synchronize(ctx)
    assert b == a + 1
    for x, y in zip(apart, once):
        kind = torch.int16 if x.element_size() == 2 else torch.int32
        assert torch.equal(torch.isnan(x), torch.isnan(y)) and torch.equal(x.nan_to_num(7).view(kind), y.nan_to_num(7).view(kind))
    assert bool(torch.isnan(apart[0]).any()) and not bool(torch.isnan(apart[0]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [128, 64, 96, 16])
def test_codes_of_all_scales_in_the_pieces(M, ctx, dtype, d):  # noqa: F811
    """Scales as test_codes_of_all_scales has them, on pages of their own in such numbers that the pieces widen codes:
    one launch less than the same batch as ordinary chunks."""
    t = Far(M, ctx, [90, 70], [2100, 1430], [2190, 1500], 8, 2, d, 16, dtype, "e4m3", seed=d, branch=6)
    g = torch.Generator(device="cuda").manual_seed(1)
    for which, (lo, hi) in ((2, (100, 128)), (3, (96, 134) if dtype == "f16" else (96, 150))):
        t.pools[which].copy_(torch.randint(lo, hi, t.pools[which].shape, generator=g, device="cuda").to(torch.uint8))
    t.pools[3][:, :, ::5] = 0
    t.pools[2][:, :, 1::7] = 0
    t.pools[2][:, :, 2::7] = 111
    t.pools[2][:, :, 3::7] = 112
    t.check()
    chain = M.mure_tokens_plan(t.cache, 8, t.new, t.pos, t.kv, t.table)
    a, b = (launches(M, ctx, t.cache, p, t.q)[0] for p in (t.plan, chain))
    M.mure_synchronize(ctx)
    assert b == a + 1
