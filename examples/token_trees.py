"""Continuations of many mutants of a network verified by the original in one pass, on token caches.

The network: token embeddings, attention blocks whose queries and keys are normed and rotated by position, and a
classifier; it continues prompts greedily.  Mutants of its classifier, run without the blocks (from the embedding of a token
alone), are cheap guesses of what it says next: from the token that the original has chosen, every mutant's guess, and the
guesses that follow those, make a tree.  One pass of the original over the tree (its tokens share the prompt's cells and
see their own ancestors) gives its choice after every guess; the path that it agrees with is kept, the rest of the tree
is killed, and the next tree grows from the path's end.  The texts are those of the original alone, whatever the
mutants say (compared with a run that chooses one token at a time).

    python examples/token_trees.py            # small, a few seconds on a GB300
    python examples/token_trees.py --prompts 64 --mutants 12 --steps 20
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


class Net:
    """Random weights of the network, fp32."""

    def __init__(self, vocab=50, layers=2, heads=4, kv_heads=2, dim=32, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.layers = heads, kv_heads, dim, layers
        width = heads * dim

        def w(*shape):
            return torch.randn(*shape, generator=g, device="cuda") / shape[-1] ** 0.5

        self.embed = torch.randn(vocab, width, generator=g, device="cuda")
        self.qkv = [w((heads + 2 * kv_heads) * dim, width) for _ in range(layers)]
        # (the blocks add little to the embedding: the guesses are then often right)
        self.o = [w(width, width) * 0.4 for _ in range(layers)]
        self.norm = 1 + 0.1 * torch.randn(2, dim, generator=g, device="cuda")
        self.out = w(vocab, width)


def guesses(net, n, seed=1):
    """[mutants][vocab]: the token that each mutant of the classifier says after a token, by the token's embedding."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    said = []
    for _ in range(n):
        out = net.out.clone()
        out[torch.randint(out.shape[0], (out.shape[0] // 4,), generator=g, device="cuda")] *= -1.0
        said.append((net.embed @ out.T).argmax(-1))
    return torch.stack(said).cpu().numpy()


class Run:
    """Prompts in token caches, one per block, continued step by step."""

    def __init__(self, ctx, net, prompts, room, page=16, form="same"):
        self.ctx, self.net = ctx, net
        pages = [-(-(len(p) + room) // page) for p in prompts]
        self.table = np.zeros((len(prompts), max(pages)), np.int32)
        for b, n in enumerate(pages):
            self.table[b, :n] = np.arange(sum(pages[:b]), sum(pages[:b]) + n)
        self.caches = [mure.mure_tokens_create(ctx, net.kv_heads, net.dim, page, sum(pages), dtype="f32", form=form) for _ in range(net.layers)]
        weights = net.norm.cpu().numpy()
        self.rotary = mure.mure_rotary_create(ctx, net.dim, q_weight=weights[0], k_weight=weights[1])
        self.held = [0] * len(prompts)
        self.plan = None
        last = self.forward(prompts, None)
        self.held = [len(p) for p in prompts]
        self.next = [c[-1] for c in last]                # the original's choice after each prompt
        self.texts = [[] for _ in prompts]

    def forward(self, tokens, parents):
        """The original's choice after each of the new tokens (lists by sequence; parents: trees)."""
        net, new = self.net, [len(t) for t in tokens]
        self.plan = mure.mure_tokens_plan(self.caches[0], net.heads, new, self.held, [a + b for a, b in zip(self.held, new)], self.table,
                                          plan=self.plan, parents=None if parents is None else [i for p in parents for i in p])
        x = net.embed[torch.tensor([t for seq in tokens for t in seq], device="cuda")]
        for i, cache in enumerate(self.caches):
            rows = (x @ net.qkv[i].T).unflatten(1, (-1, net.dim))
            q, k, v = rows.split((net.heads, net.kv_heads, net.kv_heads), 1)
            q = mure.mure_tokens_append_rotated(cache, self.plan, self.rotary, q, k, v)
            x = x + mure.mure_tokens_attend(cache, self.plan, q).flatten(1) @ net.o[i].T
        choice = (x @ net.out.T).argmax(-1).tolist()
        return [choice[sum(new[:b]):sum(new[:b + 1])] for b in range(len(new))]

    def step(self, said, depth):
        """One tree per sequence: the chosen token, the mutants' guesses after it, and so on; returns how many tokens of
        each were kept."""
        trees = []
        for t in self.next:
            tokens, parents, level = [t], [-1], [0]
            for _ in range(depth):
                below = []
                for node in level:
                    for guess in dict.fromkeys(said[:, tokens[node]].tolist()):
                        below.append(len(tokens))
                        tokens.append(guess)
                        parents.append(node)
                level = below
            trees.append((tokens, parents))
        choice = self.forward([t for t, _ in trees], [p for _, p in trees])
        kept = []
        for b, (tokens, parents) in enumerate(trees):
            path = [0]
            while True:                                  # the guess that the original agrees with, if any
                hit = [i for i in range(path[-1] + 1, len(tokens)) if parents[i] == path[-1] and tokens[i] == choice[b][path[-1]]]
                if not hit:
                    break
                path.append(hit[0])
            kept.append(path)
            self.texts[b] += [tokens[i] for i in path]
            self.next[b] = choice[b][path[-1]]
        for cache in self.caches:
            mure.mure_tokens_keep(cache, self.plan, kept)
        self.held = [n + len(path) for n, path in zip(self.held, kept)]
        return [len(path) for path in kept]


def run(prompts=12, mutants=6, steps=6, depth=2, form="same", seed=0):
    """Texts by trees and one token at a time, and how many tokens the steps kept."""
    rng = np.random.default_rng(seed)
    net = Net(seed=seed)
    said = guesses(net, mutants)
    texts = [rng.integers(0, net.embed.shape[0], rng.integers(3, 60)).tolist() for _ in range(prompts)]
    ctx = mure.mure_create(0)
    tree = mutants ** depth * 2 + mutants + 1            # room for a step's tree behind the texts
    by_tree = Run(ctx, net, texts, steps * (depth + 1) + tree, form=form)
    kept = [by_tree.step(said, depth) for _ in range(steps)]
    alone = Run(ctx, net, texts, steps * (depth + 1) + 1, form=form)
    while min(len(t) for t in alone.texts) < max(len(t) for t in by_tree.texts):
        alone.step(said, 0)
    mure.mure_synchronize(ctx)
    return {"by_tree": by_tree.texts, "alone": [a[:len(t)] for a, t in zip(alone.texts, by_tree.texts)], "kept": kept}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--prompts", type=int, default=12)
    ap.add_argument("--mutants", type=int, default=6)
    ap.add_argument("--steps", type=int, default=6)
    ap.add_argument("--form", choices=("same", "e4m3"), default="same")
    a = ap.parse_args()
    r = run(a.prompts, a.mutants, a.steps, form=a.form)
    n, kept = sum(map(len, r["by_tree"])), np.mean(r["kept"])
    same = sum(x == y for x, y in zip(r["by_tree"], r["alone"]))
    print(f"{a.prompts} prompts continued by {n} tokens, {kept:.2f} per pass of the original; {same} texts as without the mutants")
