"""Norm and rotation of queries and keys on the GPU, alone and with the write into the cells, against the formula
in 64 bits.

Tolerance, fixed by the arithmetic, with e = 2^-24 (half a step of fp32), u half a step of the output's type and
y the normed row:
  norm     the sum of squares is of one sign: 13 roundings of its chain and tree bound its relative error, halved by the
           root; rsqrt is off by 2 units in the last place (4 e), the mean's product, eps and the two
           products with the weight by one rounding each: within 6.5 + 4 + 4 < 15 e of y;
  angle    to the nearest 2^-33 of a turn, then fp32: half a step of pi v, v up to 1, is pi e; sine and cosine
           are off by one unit in the last place (2 e) beside it: within 6 e, absolutely;
  turn     two products, one of them fused: 2 e of |a| + |b|.
So an output is within u |out| + 23 e (|a| + |b|) of its value, (a, b) its pair (an unrotated one: 15 e |a|), and the type's
least step (f16: 2^-25)."""
import math
from fractions import Fraction

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_tokens import M, TYPES, UNIT, Batch, ctx  # noqa: E402,F401

E = 2.0 ** -24
TWO_PI = 2 * Fraction(31415926535897932384626433832795028841971693993751, 10 ** 49)


def turned(x, at, freq, axis, layout, weight, eps):
    """(values, tolerance but for the type's part) of rows x [n][heads][d] at positions at [axes][n], in 64 bits."""
    y = x.double().cpu()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * torch.as_tensor(weight, dtype=torch.float64)
    half, out = len(freq), y.clone()
    tol = 15 * E * y.abs()
    for i in range(half):
        a, b = (i, i + half) if layout == "halves" else (2 * i, 2 * i + 1)
        # the angle exactly, reduced to one turn
        f = Fraction(float(freq[i]))
        u = torch.tensor([float((int(p) * f / TWO_PI) % 1 * TWO_PI) for p in at[axis[i]]], dtype=torch.float64)[:, None]
        out[..., a], out[..., b] = y[..., a] * u.cos() - y[..., b] * u.sin(), y[..., b] * u.cos() + y[..., a] * u.sin()
        tol[..., a] = tol[..., b] = 23 * E * (y[..., a].abs() + y[..., b].abs())
    return out.cuda(), tol.cuda()


def near(got, want, tol, dtype):
    t = tol + UNIT[dtype] * want.abs() + (2.0 ** -25 if dtype == "f16" else 0.0) + 1e-40
    err = (got.double() - want).abs()
    assert bool((err <= t).all()), float((err / t).max())


def rotary(M, ctx, d, rot, layout, norm, axes=1, seed=0, base=10000.0):  # noqa: F811
    rng = np.random.default_rng(seed)
    freq = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    axis = [int(a) for a in rng.integers(0, axes, rot // 2)]
    w = {n: (1 + 0.3 * rng.standard_normal(d)).astype(np.float32) if n in norm else None for n in "qk"}
    r = M.mure_rotary_create(ctx, d, rot, layout=layout, freq=freq, axis=axis, n_axes=axes, q_weight=w["q"], k_weight=w["k"], eps=1e-5)
    return r, freq, axis, w


SHAPES = [(8, 2, 128, 128), (3, 1, 64, 32), (9, 3, 40, 40), (4, 2, 256, 64), (5, 5, 8, 8), (4, 2, 96, 0), (2, 1, 72, 24), (70, 2, 128, 120)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("layout", ["halves", "adjacent"])
@pytest.mark.parametrize("heads,hk,d,rot", SHAPES)
@pytest.mark.parametrize("norm", ["qk", "", "k"])
def test_rotate(M, ctx, dtype, layout, heads, hk, d, rot, norm):  # noqa: F811
    """Every type, pairing and head size, chunks of 0 to 37 tokens at the plan's positions; rows at any strides."""
    new, pos = [1, 0, 37, 5, 16], [0, 9, 3, 1000, 100]
    t = Batch(M, ctx, new, pos, [a + b for a, b in zip(new, pos)], heads, hk, d, 16, dtype, "same")
    r, freq, axis, w = rotary(M, ctx, d, rot, layout, norm)
    at = [[p + i for n, p in zip(new, pos) for i in range(n)]]
    n = len(at[0])
    qkv = torch.empty(n, heads + hk + 1, d + 3, dtype=TYPES[dtype], device="cuda")     # rows off every 16-byte boundary
    q, k = qkv[:, :heads, 1:d + 1], qkv[:, heads:heads + hk, 2:d + 2]
    q.copy_(t.q)
    k.copy_(t.k)
    before = qkv.clone()
    for a, b in ((t.q, t.k), (q, k)):
        got = M.mure_tokens_rotate(t.cache, t.plan, r, a, b)
        M.mure_synchronize(ctx)
        for x, y, name in ((t.q, got[0], "q"), (t.k, got[1], "k")):
            near(y, *turned(x, at, freq, axis, layout, w[name], 1e-5), dtype)
    M.mure_tokens_rotate(t.cache, t.plan, r, q, k, out=(q, k))                          # into the inputs
    M.mure_synchronize(ctx)
    assert torch.equal(q, got[0]) and torch.equal(k, got[1])
    q.copy_(t.q)
    k.copy_(t.k)
    assert torch.equal(qkv.view(torch.uint8), before.view(torch.uint8))                 # nothing beside them
    only = M.mure_tokens_rotate(t.cache, t.plan, r, t.q)
    assert only[1] is None and torch.equal(only[0], got[0])
    only = M.mure_tokens_rotate(t.cache, t.plan, r, k=t.k)
    assert only[0] is None and torch.equal(only[1], got[1])


@pytest.mark.parametrize("layout", ["halves", "adjacent"])
def test_positions_along_axes(M, ctx, layout):  # noqa: F811
    """Three axes of positions, each pair on one of them, over the whole range of 32 bits."""
    n, d = 33, 64
    t = Batch(M, ctx, [n], [7], [7 + n], 4, 2, d, 16, "f32", "same")
    r, freq, axis, w = rotary(M, ctx, d, d, layout, "qk", axes=3)
    rng = np.random.default_rng(1)
    at = rng.integers(-2 ** 31, 2 ** 31, (3, n))
    at[:, :5] = [[0, 1, -1, 2 ** 31 - 1, -2 ** 31]] * 3
    wide = torch.zeros(3, n + 6, dtype=torch.int32, device="cuda")
    wide[:, :n] = torch.from_numpy(at.astype(np.int32)).cuda()
    got = M.mure_tokens_rotate(t.cache, t.plan, r, t.q, t.k, positions=wide[:, :n])
    M.mure_synchronize(ctx)
    near(got[0], *turned(t.q, at, freq, axis, layout, w["q"], 1e-5), "f32")
    near(got[1], *turned(t.k, at, freq, axis, layout, w["k"], 1e-5), "f32")


@pytest.mark.parametrize("sign", [1, -1])
def test_frequencies_and_far_positions(M, ctx, sign):  # noqa: F811
    """Frequencies of either sign from 2^-40 to 2^20 radians, positions up to the last a plan takes."""
    d = 64
    t = Batch(M, ctx, [3], [5], [8], 1, 1, d, 16, "f32", "same")
    freq = [sign * 2.0 ** e * f for e, f in zip(np.linspace(-40, 19, 32), np.random.default_rng(3).uniform(1, 2, 32))]
    r = M.mure_rotary_create(ctx, d, d, freq=freq)
    plan = M.mure_tokens_plan(t.cache, 1, [3], [2 ** 30 - 3], [0], t.table)
    got = M.mure_tokens_rotate(t.cache, plan, r, t.q, t.k)
    M.mure_synchronize(ctx)
    at = [[2 ** 30 - 3 + i for i in range(3)]]
    near(got[0], *turned(t.q, at, freq, [0] * 32, "halves", None, 0), "f32")
    # the default's frequencies are those of the base
    r = M.mure_rotary_create(ctx, d, base=1e6)
    got = M.mure_tokens_rotate(t.cache, t.plan, r, t.q, t.k)
    near(got[1], *turned(t.k, [[5, 6, 7]], [1e6 ** (-2 * i / d) for i in range(d // 2)], [0] * 32, "halves", None, 0), "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e-20, 1.0, 1e18, 1e25, 1e37])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_norms_at_the_ends_of_the_range(M, ctx, dtype, size, eps):  # noqa: F811
    """Rows whose squares leave fp32's range are normed all the same."""
    d = 128
    t = Batch(M, ctx, [4], [0], [4], 2, 2, d, 16, dtype, "same")
    x = (t.q.float() * size).to(TYPES[dtype])
    w = np.ones(d, np.float32)
    r = M.mure_rotary_create(ctx, d, 0, q_weight=w, k_weight=w, eps=eps)
    got = M.mure_tokens_rotate(t.cache, t.plan, r, x, x)[0]
    M.mure_synchronize(ctx)
    assert bool(torch.isfinite(got).all())
    y = x.double()
    want = y / torch.sqrt((y * y).mean(-1, keepdim=True) + float(np.float32(eps)))
    near(got, want, 15 * E * want.abs(), dtype)


def test_zeros_infinities_and_nans(M, ctx):  # noqa: F811
    """A row of zeros stays one; a row with an infinity or a NaN is that of the formula, and its neighbours are as without."""
    d = 64
    t = Batch(M, ctx, [5], [3], [8], 2, 2, d, 16, "f32", "same")
    w = np.ones(d, np.float32)
    r = M.mure_rotary_create(ctx, d, 0, q_weight=w, k_weight=w, eps=1e-6)
    clean = M.mure_tokens_rotate(t.cache, t.plan, r, t.q, t.k)[0].clone()
    t.q[1, 0] = 0
    t.q[2, 1, 5] = math.inf
    t.q[3, 0, 9] = math.nan
    got = M.mure_tokens_rotate(t.cache, t.plan, r, t.q, t.k)[0]
    M.mure_synchronize(ctx)
    assert not bool(got[1, 0].any()) and bool(torch.isnan(got[3, 0]).all())
    assert bool(torch.isnan(got[2, 1, 5])) and not bool(got[2, 1, :5].any()) and not bool(got[2, 1, 6:].any())
    for i, h in ((0, 0), (0, 1), (1, 1), (2, 0), (3, 1), (4, 0), (4, 1)):
        assert torch.equal(got[i, h], clean[i, h])


@pytest.mark.parametrize("form", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("layout", ["halves", "adjacent"])
@pytest.mark.parametrize("heads,hk,d,rot,page", [(8, 2, 128, 128, 16), (3, 1, 64, 32, 8), (15, 5, 40, 40, 32), (4, 2, 256, 64, 64), (4, 2, 96, 0, 1024)])
def test_cells_are_those_of_the_two_calls(M, ctx, dtype, form, layout, heads, hk, d, rot, page):  # noqa: F811
    """One pass leaves the bits of a rotation and a write, in the cells and the queries, and no others."""
    new, pos = [1, 0, 37, 5, 130], [0, 9, 3, 2 * page - 2, 100]
    kv = [a + b for a, b in zip(new, pos)]
    t = Batch(M, ctx, new, pos, kv, heads, hk, d, page, dtype, form)
    u = Batch(M, ctx, new, pos, kv, heads, hk, d, page, dtype, form)
    t.k[0, 0, 1] = t.v[3, 0, 2] = math.nan
    u.k[0, 0, 1] = u.v[3, 0, 2] = math.nan
    r = rotary(M, ctx, d, rot, layout, "qk")[0]
    qa, ka = M.mure_tokens_rotate(t.cache, t.plan, r, t.q, t.k)
    M.mure_tokens_append(t.cache, t.plan, ka, t.v)
    qb = M.mure_tokens_append_rotated(u.cache, u.plan, r, u.q, u.k, u.v)
    M.mure_synchronize(ctx)
    assert torch.equal(qa, qb)
    for a, b in zip(t.pools, u.pools):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    q = u.q.clone()
    assert M.mure_tokens_append_rotated(u.cache, u.plan, r, q, u.k, u.v, out=q) is q and torch.equal(q, qa)
    for p in u.pools:
        p.view(torch.uint8).zero_()
    assert M.mure_tokens_append_rotated(u.cache, u.plan, r, None, u.k, u.v) is None
    a, b = M.mure_tokens_read(t.cache, t.plan, new=True), M.mure_tokens_read(u.cache, u.plan, new=True)
    M.mure_synchronize(ctx)
    for x, y in zip(a, b):
        assert torch.equal(x.nan_to_num(7), y.nan_to_num(7))


def test_refusals(M, ctx):  # noqa: F811
    import ctypes as C
    t = Batch(M, ctx, [2], [14], [16], 4, 2, 64, 16, "bf16", "same")
    before = [p.clone() for p in t.pools]
    w = np.ones(64, np.float32)
    r = M.mure_rotary_create(ctx, 64, q_weight=w)
    for bad in (dict(head_dim=12), dict(head_dim=0), dict(head_dim=264), dict(rot_dim=68), dict(rot_dim=72), dict(rot_dim=-8), dict(n_axes=0),
                dict(n_axes=9), dict(base=0.0), dict(base=math.nan), dict(eps=-1.0), dict(eps=math.nan), dict(eps=2.0),
                dict(freq=[math.inf] * 32), dict(freq=[2.0 ** 21] * 32), dict(axis=[1] * 32)):
        with pytest.raises(M.MureError) as ei:
            M.mure_rotary_create(ctx, **{**dict(head_dim=64, rot_dim=64 if "head_dim" not in bad else bad["head_dim"]), **bad})
        assert ei.value.status == 1, bad
    for bad in (dict(freq=[1.0] * 31), dict(axis=[0] * 33), dict(axis=[-1] * 32), dict(axis=[256] * 32), dict(q_weight=w[:63])):
        with pytest.raises(ValueError):
            M.mure_rotary_create(ctx, 64, **bad)
    d = M._RotaryDesc(64, 64, 2, 1, None, 1e4, None, None, None, 0.0, 0)
    assert M.lib().mure_rotary_create(ctx.h, C.byref(d), C.byref(C.c_void_p())) == 2
    d = M._RotaryDesc(64, 64, 0, 1, None, 1e4, None, None, None, 0.0, 1)
    assert M.lib().mure_rotary_create(ctx.h, C.byref(d), C.byref(C.c_void_p())) == 1
    other = M.mure_create(0)
    for wrong in (M.mure_rotary_create(ctx, 128), M.mure_rotary_create(other, 64)):
        for call in (lambda: M.mure_tokens_rotate(t.cache, t.plan, wrong, t.q, t.k),
                     lambda: M.mure_tokens_append_rotated(t.cache, t.plan, wrong, t.q, t.k, t.v)):
            with pytest.raises(M.MureError) as ei:
                call()
            assert ei.value.status == 1
    at = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    for bad in (at.cpu(), at.long(), at[:, :1], torch.zeros(2, 2, dtype=torch.int32, device="cuda"),
                torch.zeros(1, 4, dtype=torch.int32, device="cuda")[:, ::2]):
        with pytest.raises(ValueError):
            M.mure_tokens_rotate(t.cache, t.plan, r, t.q, t.k, positions=bad)
    for bad in (t.q.float(), t.q[:1], t.q.cpu(), t.q.clone().requires_grad_()):
        with pytest.raises(ValueError):
            M.mure_tokens_rotate(t.cache, t.plan, r, bad, t.k)
    with pytest.raises(ValueError):
        M.mure_tokens_rotate(t.cache, t.plan, r, t.q, out=(t.q, t.k))
    L, rows, ref = M.lib(), M._TokensRows, C.byref
    out = torch.zeros_like(t.q)
    q, o = rows(t.q.data_ptr(), 256, 64), rows(out.data_ptr(), 256, 64)
    k, v = rows(t.k.data_ptr(), 128, 64), rows(t.v.data_ptr(), 128, 64)
    odd, same = rows(t.q.data_ptr() + 1, 256, 64), rows(out.data_ptr(), 0, 64)
    call = lambda *a: L.mure_tokens_rotate(t.cache.h, t.plan.h, r.h, *a)  # noqa: E731
    assert call(None, 0, ref(q), None, ref(o), None) == 0
    for bad in ((None, 0, ref(q), None, None, None), (None, 0, None, None, ref(o), None), (None, 0, ref(odd), None, ref(o), None),
                (None, 0, ref(q), None, ref(same), None), (at.data_ptr(), 1, ref(q), None, ref(o), None),
                (at.data_ptr() + 2, 2, ref(q), None, ref(o), None), (None, 0, ref(rows(None, 1, 1)), None, ref(o), None)):
        assert call(*bad) == 1
    out.zero_()
    put = lambda *a: L.mure_tokens_append_rotated(t.cache.h, t.plan.h, r.h, *a)  # noqa: E731
    for bad in ((None, 0, ref(q), ref(k), None, ref(o)), (None, 0, ref(q), None, ref(v), ref(o)), (None, 0, ref(q), ref(k), ref(v), None)):
        assert put(*bad) == 1
    assert L.mure_tokens_rotate(t.cache.h, t.plan.h, None, None, 0, ref(q), None, ref(o), None) == 1
    assert L.mure_tokens_rotate(t.cache.h, None, r.h, None, 0, ref(q), None, ref(o), None) == 1
    p = M.mure_tokens_plan(t.cache, 4, [2], [15], [16], t.table)                    # past the cells: rotated, not written
    M.mure_tokens_rotate(t.cache, p, r, t.q, t.k)
    with pytest.raises(M.MureError):
        M.mure_tokens_append_rotated(t.cache, p, r, t.q, t.k, t.v)
    M.mure_synchronize(ctx)
    assert not bool(out.any()) and all(torch.equal(a, b) for a, b in zip(before, t.pools))
