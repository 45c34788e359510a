"""Memoized mutation testing of a network that attends over tokens, on token caches.

The network: token embeddings, one attention block per layer (queries, keys, values and an output
projection, added to the block's input), and a classifier on the last token.  The original runs once over
every input and leaves each layer's keys and values in a token cache.  Mutants of the last
block's queries or output projection and of the classifier leave those keys and values as they are: a
mutant's sequence names the original's pages in its table, and only the last token's query attends
again, all mutants and all inputs in one call (or in several of 65,535 sequences).  The same mutants run
end to end without any cache, in plain torch, for comparison.

    python examples/token_mutants.py            # small, a few seconds on a GB300
    python examples/token_mutants.py --inputs 200 --mutants 100 --form e4m3
"""
import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2607_18582_gb300 import mure  # noqa: E402

SEQS = 65_535        # sequences of a plan, at most


class Net:
    """Random weights of the network, fp32."""

    def __init__(self, vocab=200, layers=2, heads=8, kv_heads=2, dim=32, classes=10, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.layers = heads, kv_heads, dim, layers
        width = heads * dim

        def w(*shape):
            return torch.randn(*shape, generator=g, device="cuda") / shape[-1] ** 0.5

        self.embed = torch.randn(vocab, width, generator=g, device="cuda")
        self.q = [w(width, width) for _ in range(layers)]
        self.k = [w(kv_heads * dim, width) for _ in range(layers)]
        self.v = [w(kv_heads * dim, width) for _ in range(layers)]
        self.o = [w(width, width) for _ in range(layers)]
        self.out = w(classes, width)


def mutants(net, n, seed=1):
    """(which weights, neuron, operator): a neuron of the last block's queries or output projection, or of the
    classifier, is held at 0 (NEB) or negated (NAI)."""
    rng = np.random.default_rng(seed)
    rows = []
    for i in range(n):
        where = ("q", "o", "out")[i % 3]
        rows.append((where, int(rng.integers(net.out.shape[0] if where == "out" else net.o[0].shape[0])),
                     ("NEB", "NAI")[int(rng.integers(2))]))
    return rows


def mutated(net, mutant):
    """The last block's (queries, output projection) and the classifier of a mutant."""
    w = {"q": net.q[-1], "o": net.o[-1], "out": net.out}
    where, j, op = mutant
    w[where] = w[where].clone()
    w[where][j] *= 0.0 if op == "NEB" else -1.0
    return w["q"], w["o"], w["out"]


class Memo:
    """The original's run over the inputs, with its caches."""

    def __init__(self, ctx, net, tokens, lengths, page=16, form="same"):
        self.ctx, self.net, self.lengths = ctx, net, lengths
        pages = [-(-n // page) for n in lengths]
        self.table = np.zeros((len(lengths), max(pages)), np.int32)
        for b, n in enumerate(pages):
            self.table[b, :n] = np.arange(sum(pages[:b]), sum(pages[:b]) + n)
        self.caches = [mure.mure_tokens_create(ctx, net.kv_heads, net.dim, page, sum(pages), dtype="f32", form=form)
                       for _ in range(net.layers)]
        x = net.embed[tokens]                                   # the inputs' tokens, one after the other
        plans, at = [], 0                                       # every layer's: (rows, plan) of up to SEQS inputs
        for i in range(0, len(lengths), SEQS):
            part = lengths[i:i + SEQS]
            plans.append((slice(at, at + sum(part)), mure.mure_tokens_plan(self.caches[0], net.heads, part, [0] * len(part), part,
                                                                           self.table[i:i + SEQS])))
            at += sum(part)
        for i, cache in enumerate(self.caches):
            last = i == net.layers - 1
            if last:
                self.x = x
            rows = [(x @ w.T).unflatten(1, (-1, net.dim)) for w in (net.q[i], net.k[i], net.v[i])]
            a = torch.empty_like(rows[0])
            for r, plan in plans:
                mure.mure_tokens_append(cache, plan, rows[1][r], rows[2][r])
                mure.mure_tokens_attend(cache, plan, rows[0][r], out=a[r])
            x = x + a.flatten(1) @ net.o[i].T
        ends = torch.tensor(np.cumsum(lengths) - 1, device="cuda")
        self.x = self.x[ends]                                   # the last block's input at each last token
        self.pred = (x[ends] @ net.out.T).argmax(-1)

    def kills(self, mutants_):
        """Kill matrix [mutants][inputs]: only the last token's query attends again, over shared pages."""
        net, n, m = self.net, len(self.lengths), len(mutants_)
        w = [mutated(net, u) for u in mutants_]
        q = torch.stack([self.x @ wq.T for wq, _, _ in w]).reshape(m * n, net.heads, net.dim)
        a = torch.empty_like(q)
        lengths = np.asarray(self.lengths, np.int32)
        for i in range(0, m * n, SEQS):
            part = np.arange(i, min(i + SEQS, m * n)) % n       # the inputs of these (mutant, input) pairs
            plan = mure.mure_tokens_plan(self.caches[-1], net.heads, np.ones(len(part), np.int32), lengths[part] - 1, lengths[part],
                                         self.table[part])
            mure.mure_tokens_attend(self.caches[-1], plan, q[i:i + SEQS], out=a[i:i + SEQS])
        a = a.reshape(m, n, -1)
        logits = torch.stack([(self.x + a[i] @ wo.T) @ wc.T for i, (_, wo, wc) in enumerate(w)])
        return logits.argmax(-1) != self.pred, logits

    def cells(self):
        """The last block's keys and values as its mutants see them, dense (inputs one after the other)."""
        parts = []
        for i in range(0, len(self.lengths), SEQS):
            held = self.lengths[i:i + SEQS]
            zero = [0] * len(held)
            plan = mure.mure_tokens_plan(self.caches[-1], self.net.heads, zero, zero, held, self.table[i:i + SEQS])
            parts.append(mure.mure_tokens_read(self.caches[-1], plan))
        return tuple(torch.cat(x) for x in zip(*parts))


def vanilla_logits(net, mutant, tokens, lengths):
    """A mutant end to end, no cache, 64-bit sums (plain fp32 cells)."""
    wq, wo, wc = (t.double() for t in mutated(net, mutant))
    rows, at = [], 0
    for n in lengths:
        x = net.embed[tokens[at:at + n]].double()
        at += n
        for i in range(net.layers):
            last = i == net.layers - 1
            q = (x @ (wq if last else net.q[i].double()).T).unflatten(1, (net.heads, net.dim))
            k, v = ((x @ u[i].double().T).unflatten(1, (net.kv_heads, net.dim)).repeat_interleave(net.heads // net.kv_heads, 1)
                    for u in (net.k, net.v))
            s = torch.einsum("qhd,khd->hqk", q, k) / net.dim ** 0.5
            s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=s.device).triu(1), -float("inf"))
            a = torch.einsum("hqk,khd->qhd", s.softmax(-1), v).flatten(1)
            x = x + a @ (wo if last else net.o[i].double()).T
        rows.append(x[-1] @ wc.T)
    return torch.stack(rows)


def run(inputs=40, n_mutants=30, form="same", seed=0):
    """Kill matrices of the memoized and the vanilla run, and the vanilla logits' margins."""
    rng = np.random.default_rng(seed)
    net = Net(seed=seed)
    lengths = [int(n) for n in rng.integers(5, 120, inputs)]
    tokens = torch.from_numpy(rng.integers(0, net.embed.shape[0], sum(lengths))).cuda()
    ctx = mure.mure_create(0)
    memo = Memo(ctx, net, tokens, lengths, form=form)
    table = mutants(net, n_mutants)
    kill, logits = memo.kills(table)
    mure.mure_synchronize(ctx)
    exact = torch.stack([vanilla_logits(net, u, tokens, lengths) for u in table])
    top = exact.topk(2, -1).values
    return {"kill": kill, "logits": logits, "vanilla": exact.argmax(-1) != memo.pred, "exact": exact,
            "margin": top[..., 0] - top[..., 1], "memo": memo}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--inputs", type=int, default=40)
    ap.add_argument("--mutants", type=int, default=30)
    ap.add_argument("--form", choices=("same", "e4m3"), default="same")
    a = ap.parse_args()
    r = run(a.inputs, a.mutants, a.form)
    off = (r["logits"] - r["exact"]).abs().max().item()
    print(f"{a.mutants} mutants x {a.inputs} inputs: {int(r['kill'].sum())} kills memoized, {int(r['vanilla'].sum())} vanilla, "
          f"{int((r['kill'] != r['vanilla']).sum())} differ; logits off by {off:.2g}")
