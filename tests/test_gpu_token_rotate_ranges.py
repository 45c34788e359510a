"""The norm and rotation at the ends of their ranges on the GPU: rows whose squares leave fp32,
angles beside a quarter turn's multiples, and batches of more tiles than blocks that run at a time.  Tolerances as in test_gpu_token_rotate.py, but for the angles.

There sine or cosine is small, and its relative error counts, e = 2^-24: the angle's fraction of a turn is right to 2 units
of 2^-64 for each position; its nearest multiple of 2^-32 goes to sine and cosine (2 e), which what is left, at most half
of that multiple or all there is, corrects to the first order: three roundings (its own, pi's and the
product's) and one of the sum, in which at most half of the sine is cancelled: within 2 (2 + 3) + 1 = 11 e; the product with
the value one more."""
import math
from fractions import Fraction

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_token_rotate import E, TWO_PI, near, rotary, turned  # noqa: E402
from test_gpu_tokens import M, TYPES, Batch, ctx  # noqa: E402,F401


def normed(M, ctx, x, dtype, eps):  # noqa: F811
    """Rows [n][2][d] normed, not rotated, and the formula's in 64 bits."""
    n, _, d = x.shape
    t = Batch(M, ctx, [n], [0], [n], 2, 2, d, 16, dtype, "same")
    w = np.ones(d, np.float32)
    r = M.mure_rotary_create(ctx, d, 0, q_weight=w, k_weight=w, eps=eps)
    got = M.mure_tokens_rotate(t.cache, t.plan, r, x, x)
    M.mure_synchronize(ctx)
    assert torch.equal(got[0], got[1])
    y = x.double()
    return got[0], y / torch.sqrt((y * y).mean(-1, keepdim=True) + float(np.float32(eps)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [3e-45, 1e-44, 3e-42, 1e-40, 1.3 * 2.0 ** -130, 2.0 ** -126, 1e-36, 1e-25, 1e-12, 3e38])
@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-38, 7e-31, 9e-31, 1e-6])
def test_norms_of_any_size(M, ctx, dtype, size, eps):  # noqa: F811
    """Rows down to fp32's least numbers, random, constant, and with one value that is not zero; where eps is
    nothing beside them, or all there is."""
    d = 128
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.rand(6, 2, d, generator=g, device="cuda", dtype=torch.float64) * 2 - 1
    x[2] = 1.0
    x[3] = -0.75
    x[4] = 0.0
    x[4, :, 77] = 1.0
    x[5] = 0.0
    x[5, :, 3] = -0.6
    x[5, :, 100] = 0.9
    x = (x * size).float().to(TYPES[dtype])
    if dtype == "bf16":
        x = torch.where(x.abs().amax(-1, keepdim=True) == 0, torch.full_like(x, 2.0 ** -133), x)     # (its least number)
    got, want = normed(M, ctx, x, dtype, eps)
    assert bool(torch.isfinite(got).all())
    near(got, want, 15 * E * want.abs(), dtype)


def test_norms_of_values_far_apart(M, ctx):  # noqa: F811
    """Small values beside ones whose squares leave fp32 keep their bits."""
    x = torch.zeros(3, 2, 64, device="cuda")
    x[0, :, ::3] = 2.0 ** 62
    x[0, :, 1] = 1.3 * 2.0 ** -60
    x[1, :, 5] = 3e38
    x[1, :, 6] = 1.7
    x[2, :, 7] = 2.0 ** -100
    x[2, :, 8] = 1.9 * 2.0 ** -126
    got, want = normed(M, ctx, x, "f32", 0.0)
    err = (got.double() - want).abs()
    assert bool((err <= 16 * E * want.abs() + 2.0 ** -149).all()), (err / want.abs()).nan_to_num(0).max()


@pytest.mark.parametrize("layout", ["halves", "adjacent"])
@pytest.mark.parametrize("quarters", [0, 1, 2, 3])
@pytest.mark.parametrize("position", [1, -3, 1000, 2 ** 30])
def test_angles_beside_quarter_turns(M, ctx, layout, quarters, position):  # noqa: F811
    """A pair whose other value is 0 keeps fp32's relative bits however near its angle lies to a multiple of a quarter turn."""
    d, half, e = 64, 32, 2.0 ** -24
    # quarters of a turn at that position, and 2^-50 to 2^-3 radians of either sign beside them
    beside = [(-1) ** i * 2.0 ** x * 1.3 for i, x in enumerate(np.linspace(-50, -3, half))]
    freq = [float((TWO_PI * quarters / 4 + Fraction(b)) / position) for b in beside]
    r = M.mure_rotary_create(ctx, d, d, layout=layout, freq=freq)
    t = Batch(M, ctx, [2], [0], [2], 1, 1, d, 16, "f32", "same")
    first = [i for i in range(half)] if layout == "halves" else [2 * i for i in range(half)]
    second = [i + half for i in range(half)] if layout == "halves" else [2 * i + 1 for i in range(half)]
    x = torch.zeros(2, 1, d, device="cuda")
    x[0, 0, first], x[1, 0, second] = 1.5, 1.5
    at = torch.full((1, 2), position, dtype=torch.int32, device="cuda")
    got = M.mure_tokens_rotate(t.cache, t.plan, r, x, positions=at)[0].double().cpu()
    M.mure_synchronize(ctx)
    for i in range(half):
        # what is left of the angle beside the nearest quarter turn, exactly
        angle = position * Fraction(freq[i])
        q = round(angle / TWO_PI * 4)
        left = float(angle - q * TWO_PI / 4)
        s, c = [(math.sin(left), math.cos(left)), (math.cos(left), -math.sin(left)),
                (-math.sin(left), -math.cos(left)), (-math.cos(left), math.sin(left))][q % 4]
        tol = 14 * e * 1.5 + 2.0 ** -64 * 2 * abs(position) * 2 * math.pi * 1.5 / min(abs(s), abs(c))       # of either one
        for row, a, b in ((0, c, s), (1, -s, c)):
            for j, v in ((first[i], a), (second[i], b)):
                assert abs(float(got[row, 0, j]) - 1.5 * v) <= tol * abs(v) + 1e-45, (i, row, v, float(got[row, 0, j]) / (1.5 * v))


@pytest.mark.parametrize("dtype,form", [("bf16", "e4m3"), ("f16", "same"), ("f32", "same")])
@pytest.mark.parametrize("layout", ["halves", "adjacent"])
def test_more_tiles_than_blocks(M, ctx, dtype, form, layout):  # noqa: F811
    """Prompts in numbers: a block then takes all heads of its tile.  Rows are the formula's, those of a batch of a few of the
    sequences, and what the two calls store."""
    n, heads, hk, d, rot = 700, 12, 3, 64, 16
    new, pos = [1 + 7 * b % 45 for b in range(n)], [3 * b % 50 for b in range(n)]
    kv = [a + b for a, b in zip(new, pos)]
    assert sum(-(-x // 16) for x in new) > 4 * 152
    t = Batch(M, ctx, new, pos, kv, heads, hk, d, 16, dtype, form)
    r, freq, axis, w = rotary(M, ctx, d, rot, layout, "qk")
    q, k = M.mure_tokens_rotate(t.cache, t.plan, r, t.q, t.k)
    M.mure_synchronize(ctx)
    at = [[p + i for a, p in zip(new, pos) for i in range(a)]]
    near(q, *turned(t.q, at, freq, axis, layout, w["q"], 1e-5), dtype)
    near(k, *turned(t.k, at, freq, axis, layout, w["k"], 1e-5), dtype)
    few = 9
    rows = sum(new[:few])
    plan = M.mure_tokens_plan(t.cache, heads, new[:few], pos[:few], kv[:few], t.table)
    a, b = M.mure_tokens_rotate(t.cache, plan, r, t.q[:rows], t.k[:rows])
    M.mure_synchronize(ctx)
    assert torch.equal(a, q[:rows]) and torch.equal(b, k[:rows])
    for p in t.pools:
        p.view(torch.uint8).zero_()
    M.mure_tokens_append(t.cache, t.plan, k, t.v)
    want = [p.clone() for p in t.pools]
    for p in t.pools:
        p.view(torch.uint8).zero_()
    got = M.mure_tokens_append_rotated(t.cache, t.plan, r, t.q, t.k, t.v)
    M.mure_synchronize(ctx)
    assert torch.equal(got, q)
    for x, y in zip(t.pools, want):
        assert bool(y.view(torch.uint8).any()) and torch.equal(x.view(torch.uint8), y.view(torch.uint8))
