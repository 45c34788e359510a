"""The token-mutant example: memoized kills on shared pages equal the vanilla ones, fp32 logits agree with
64-bit ones, and timed-out waits of the tensor-core attention are reported and survived."""
import os
import sys

import numpy as np
import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def M():
    from paper_2607_18582_gb300 import build
    build.build()
    from paper_2607_18582_gb300 import mure
    return mure


@pytest.fixture(scope="module")
def example(M):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import token_mutants
    return token_mutants


def test_memoized_kills_equal_vanilla(example):
    """fp32 cells: logits within 1e-4 of the largest (the library's bound for fp32 networks), kills equal
    wherever the vanilla margin is not a near tie of that size."""
    r = example.run(inputs=37, n_mutants=24)
    scale = r["exact"].abs().amax(-1, keepdim=True)
    assert bool(((r["logits"] - r["exact"]).abs() <= 1e-4 * scale).all())
    near = r["margin"] < 2e-4 * scale[..., 0]
    assert bool(((r["kill"] == r["vanilla"]) | near).all())
    assert 0 < int(r["kill"].sum()) < r["kill"].numel()


def test_quantised_cells_are_what_the_mutants_see(example):
    """e4m3 cells: the memoized logits equal those of the dense cells that the cache gives back."""
    r = example.run(inputs=20, n_mutants=9, form="e4m3")
    memo = r["memo"]
    net, (k, v) = memo.net, (t.double() for t in memo.cells())
    table = example.mutants(net, 9)
    for i, u in enumerate(table):
        wq, wo, wc = (t.double() for t in example.mutated(net, u))
        at = 0
        for b, n in enumerate(memo.lengths):
            x = memo.x[b].double()
            q = (x @ wq.T).view(net.heads, net.dim)
            kk, vv = (t[at:at + n].repeat_interleave(net.heads // net.kv_heads, 1) for t in (k, v))
            at += n
            p = (torch.einsum("hd,khd->hk", q, kk) / net.dim ** 0.5).softmax(-1)
            logits = (x + torch.einsum("hk,khd->hd", p, vv).flatten() @ wo.T) @ wc.T
            assert bool(((r["logits"][i, b] - logits).abs() <= 1e-4 * logits.abs().max()).all())


def test_expired_waits_are_reported_and_the_context_recovers(M):
    """The chunk kernel's waits are bounded: with a limit of one cycle they give up, mure_synchronize
    reports it once, and with the default limit back the same bits come out as before."""
    ctx = M.mure_create(0)
    cache = M.mure_tokens_create(ctx, 2, 128, 16, 60, dtype="bf16")
    plan = M.mure_tokens_plan(cache, 8, [300, 5], [500, 40], [800, 45], np.arange(120, dtype=np.int32).reshape(2, 60) % 60)
    g = torch.Generator(device="cuda").manual_seed(0)
    q = torch.randn(305, 8, 128, generator=g, device="cuda").bfloat16()
    fill = M.mure_tokens_plan(cache, 8, [960], [0], [960], np.arange(60, dtype=np.int32)[None])
    M.mure_tokens_append(cache, fill, *(torch.randn(960, 2, 128, generator=g, device="cuda").bfloat16() for _ in range(2)))
    ref = M.mure_tokens_attend(cache, plan, q, lse=True)
    M.mure_synchronize(ctx)
    M.mure_set_wait_limit(ctx, 1)
    M.mure_tokens_attend(cache, plan, q)
    with pytest.raises(M.MureError) as ei:
        M.mure_synchronize(ctx)
    assert ei.value.status == 5
    M.mure_set_wait_limit(ctx, 0)
    M.mure_synchronize(ctx)
    again = M.mure_tokens_attend(cache, plan, q, lse=True)
    M.mure_synchronize(ctx)
    assert torch.equal(again[0], ref[0]) and torch.equal(again[1], ref[1])
