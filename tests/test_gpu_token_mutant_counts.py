"""The token-mutant example with more (mutant, input) pairs than a plan has sequences, and more inputs."""
import numpy as np
import pytest

from test_gpu_token_mutants import M, example  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def memo_of(M, example, inputs):  # noqa: F811
    rng = np.random.default_rng(3)
    net = example.Net(seed=3)
    lengths = [int(n) for n in rng.integers(3, 12, inputs)]
    tokens = torch.from_numpy(rng.integers(0, net.embed.shape[0], sum(lengths))).cuda()
    return net, tokens, lengths, example.Memo(M.mure_create(0), net, tokens, lengths)


def test_pairs_past_one_plan(M, example):  # noqa: F811
    """230 mutants x 300 inputs: as the mutants by themselves, in the library's bound for fp32 networks."""
    net, _, _, memo = memo_of(M, example, 300)
    table = example.mutants(net, 230)
    assert len(table) * 300 > 65535
    kill, logits = memo.kills(table)
    for i in (0, 100, 217, 218, 219, 229):
        k, x = memo.kills(table[i:i + 1])
        scale = x.abs().amax(-1, keepdim=True)
        assert bool(((logits[i] - x[0]).abs() <= 1e-4 * scale[0]).all())
        top = x.topk(2, -1).values
        near = top[..., 0] - top[..., 1] < 2e-4 * scale[..., 0]
        assert bool(((kill[i] == k[0]) | near[0]).all())


def test_inputs_past_one_plan(M, example, monkeypatch):  # noqa: F811
    """Inputs in several plans (of 64 here): predictions and kills as with one."""
    net, tokens, lengths, memo = memo_of(M, example, 150)
    table = example.mutants(net, 3)
    kill, logits = memo.kills(table)
    monkeypatch.setattr(example, "SEQS", 64)
    parts = example.Memo(M.mure_create(0), net, tokens, lengths)
    assert bool(((parts.x - memo.x).abs() <= 1e-4 * memo.x.abs().amax(-1, keepdim=True)).all())
    _, other = parts.kills(table)
    assert bool(((logits - other).abs() <= 1e-4 * logits.abs().amax(-1, keepdim=True)).all())
    for a, b in zip(parts.cells(), memo.cells()):
        assert a.shape == b.shape and bool(((a - b).abs() <= 1e-4 * b.abs().amax()).all())
