"""The example of trees on e4m3 cells on the GPU, by its values: what its caches hold, and every choice it makes."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from conftest import ROOT  # noqa: E402
from test_gpu_tokens import M  # noqa: E402,F401


def rotated(x, at, weight):
    """Rows [tokens][heads][d] normed and rotated, pairs of halves, in 64 bits."""
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + float(np.float32(1e-6))) * weight
    half = x.shape[-1] // 2
    freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=x.device) / half)
    u = (at[:, None] * freq)[:, None]
    a, b = y[..., :half], y[..., half:]
    return torch.cat((a * u.cos() - b * u.sin(), b * u.cos() + a * u.sin()), -1)


def test_the_example_on_e4m3_cells(M):  # noqa: F811
    """What the example's caches hold, and every choice it makes, against its network in 64 bits over those cells.

    A cell is off its value by half a step of its code, 2^-4 of it (or below the normal codes by 2^-10 of the scale, which is at
    most twice the row's largest value / 448), or a little more where fp32 rounds to the other side: 2^-4 (1 + 2^-10).  A choice's
    logit lies no further below the largest one than fp32's errors: some ten products in a chain, each of up to
    256 terms, 256 2^-24 (sum of magnitudes, below 12) each, twice: 10 * 256 * 2^-24 * 12 * 2 < 4e-3."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import token_trees as example
    ctx = M.mure_create(0)  # noqa: F811
    net = example.Net(seed=0)
    said = example.guesses(net, 6)
    rng = np.random.default_rng(4)
    texts = [rng.integers(0, 50, k).tolist() for k in (3, 20, 41, 60)]
    r = example.Run(ctx, net, texts, 4 * 3 + 80, form="e4m3")
    kept = [r.step(said, 2) for _ in range(4)]
    assert max(map(max, kept)) > 1
    plan = M.mure_tokens_plan(r.caches[0], net.heads, [0] * 4, [0] * 4, r.held, r.table)
    cells = [[x.double() for x in M.mure_tokens_read(c, plan)] for c in r.caches]
    M.mure_synchronize(ctx)
    wide = lambda x: x.double()  # noqa: E731
    g, row = net.heads // net.kv_heads, 0
    for b, prompt in enumerate(texts):
        tokens = prompt + r.texts[b]
        n = len(tokens)
        assert r.held[b] == n
        x, at = wide(net.embed)[tokens], torch.arange(n, dtype=torch.float64, device="cuda")
        mask = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        for i in range(net.layers):
            q, k, v = (x @ wide(net.qkv[i]).T).unflatten(1, (-1, net.dim)).split((net.heads, net.kv_heads, net.kv_heads), 1)
            q, k = rotated(q, at, wide(net.norm)[0]), rotated(k, at, wide(net.norm)[1])
            kc, vc = (c[row:row + n] for c in cells[i])
            for got, want in ((kc, k), (vc, v)):
                most = want.abs().amax(-1, keepdim=True)
                assert bool(((got - want).abs() <= 2.0 ** -4 * (1 + 2.0 ** -10) * want.abs() + 2.0 ** -10 * most / 224 * 1.001 + 1e-6).all())
            s = torch.einsum("ihd,jhd->hij", q, kc.repeat_interleave(g, 1)) * net.dim ** -0.5
            p = torch.softmax(s.masked_fill(~mask, -torch.inf), -1)
            x = x + torch.einsum("hij,jhd->ihd", p, vc.repeat_interleave(g, 1)).flatten(1) @ wide(net.o[i]).T
        row += n
        logits = (x @ wide(net.out).T)[len(prompt) - 1:]
        choice = torch.tensor(r.texts[b] + [r.next[b]], device="cuda")
        assert bool((logits.gather(1, choice[:, None])[:, 0] >= logits.amax(-1) - 4e-3).all())
