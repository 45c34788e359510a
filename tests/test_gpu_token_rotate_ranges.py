"""The norm and rotation at the ends of their ranges on the GPU: rows whose squares leave fp32.  Tolerances as in
test_gpu_token_rotate.py."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_token_rotate import E, near  # noqa: E402
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
