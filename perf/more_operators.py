"""A step over trees of drafted tokens on a paged token cache, as cases that can be timed and checked.

The continuations of one sequence (of the mutants of a network, or drafts of a smaller one) share
its earlier tokens and diverge as a tree.  Their new tokens pass through

  rotate  a norm of each head's query and key and the rotation by the token's position (one or
          several axes), in one pass;
  place   the same pass, which also writes the keys and the values into their cells;
  tree    attention of the tree's tokens over the sequence's earlier cells and their own ancestors;
  step    place, tree, and the cells of one path of the tree moved up to follow the earlier ones;
  fork    pages copied, so that a second sequence continues from them.

Fields of a case: `op`; `n_seqs` sequences with `past_lo` .. `past_hi` tokens in the cache and
`new_lo` .. `new_hi` new ones (both spread over the sequences by a fixed rule; fork: the sequences'
last `new_hi` pages are copied); `heads` query heads on `kv_heads` cached ones, of `dim` values;
`page` cells per page; `dtype` of the activations; `form` of the cells ("same" or "e4m3"); `window`
(0: none) and `sinks`; `rot` rotated values of a head, in pairs as `layout` says ("halves" or
"adjacent"), over `axes` axes of positions; `norm`: whether q and k are normed; `branch`: a new
token's parent is one of the `branch` tokens before it (1: a chain, 0: no tree, a chunk).
"""
import math
import random

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_EPS = 1e-6
_BASE = 500000.0


def _case(op, n_seqs, past, new, heads, kv_heads, dim, page, dtype, form="same", window=0, sinks=0, rot=0, layout="halves",
          axes=1, norm=False, branch=0):
    return {"op": op, "n_seqs": n_seqs, "past_lo": past[0], "past_hi": past[1], "new_lo": new[0], "new_hi": new[1],
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype, "form": form,
            "window": window, "sinks": sinks, "rot": rot, "layout": layout, "axes": axes, "norm": norm, "branch": branch}


def listed():
    def named(name, *a, **k):
        return dict(_case(*a, **k), name=name)

    return [
        # a decoding step of a small batch: a token per sequence, the launch counts
        named("rotate_token", "rotate", 48, (100, 4000), (1, 1), 32, 8, 128, 16, "bf16", rot=128, norm=True),
        # patches of images of different sizes: time, height and width, heads of 80 values, no norm
        named("rotate_axes", "rotate", 9, (0, 0), (1001, 5003), 16, 16, 80, 16, "f16", rot=80, layout="adjacent", axes=3),
        # a decoding step of many sequences, into their cells
        named("place_token", "place", 200, (30, 900), (1, 1), 32, 8, 128, 16, "bf16", rot=128, norm=True),
        # the prompts of a test set entering a quantised cache (what is stored is read back, as its readers see it)
        named("place_prompts_e4m3", "place", 24, (0, 0), (500, 4100), 32, 8, 128, 16, "bf16", "e4m3", rot=128, norm=True),
        # one sequence, a small tree: the latency of a single answer
        named("tree_one", "tree", 1, (700, 700), (24, 24), 32, 8, 128, 16, "bf16", branch=6),
        # trees over many quantised sequences of different lengths
        named("tree_batch_e4m3", "tree", 48, (500, 6000), (17, 64), 32, 8, 128, 16, "bf16", "e4m3", branch=8),
        # two long documents
        named("tree_long", "tree", 2, (100001, 131071), (50, 64), 32, 8, 128, 64, "bf16", branch=10),
        # trees within a window and the first tokens, odd head counts
        named("tree_window", "tree", 64, (300, 9000), (3, 40), 15, 5, 64, 16, "f16", window=1024, sinks=4, branch=5),
        # one step: rotated, stored, attended, and the accepted path kept
        named("step_batch", "step", 24, (700, 3000), (30, 64), 32, 8, 128, 16, "bf16", rot=128, norm=True, branch=8),
        # the same in the fp32 of this framework's own networks, part of a head rotated
        named("step_f32", "step", 8, (0, 900), (1, 33), 12, 4, 64, 16, "f32", rot=32, norm=True, branch=4),
        # the last page of each sequence copied for a second one that continues there
        named("fork_last", "fork", 64, (200, 500), (1, 1), 32, 8, 128, 16, "bf16"),
        # whole sequences copied
        named("fork_all", "fork", 48, (4000, 5000), (125, 250), 32, 8, 128, 16, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    while True:
        op = rng.choice(["rotate", "place", "tree", "tree", "step", "fork"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        form = rng.choice(["same", "e4m3"]) if op in ("place", "tree") else "same"
        kv_heads = rng.choice([1, 2, 3, 4, 5, 8])
        heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 8])
        dim = rng.choice([32, 40, 64, 64, 80, 96, 128, 128, 128])
        page = rng.choice([8, 16, 16, 32, 64, 128])
        window, sinks, branch = 0, 0, 0
        rot = rng.choice([dim, dim, dim - 8, max(8, dim // 16 * 8)])
        layout, axes, norm = rng.choice(["halves", "halves", "adjacent"]), rng.choice([1, 1, 2, 3]), rng.random() < 0.6
        if op in ("rotate", "place"):
            n = _log_int(rng, 1, 200)
            new_hi = 1 if rng.random() < 0.4 else _log_int(rng, 2, 4100)
            new = (max(1, new_hi // rng.choice([1, 3, 20])), new_hi)
            past_hi = _log_int(rng, 1, 2000)
            past = (rng.randint(0, past_hi), past_hi)
        elif op in ("tree", "step"):
            n = _log_int(rng, 1, 64)
            new_hi = _log_int(rng, 1, 200)
            new = (rng.randint(1, new_hi), new_hi)
            past_hi = _log_int(rng, 10, 100000 if op == "tree" else 6000)
            past = (rng.randint(0, past_hi), past_hi)
            branch = rng.choice([1, 2, 4, 8, 16])
            if rng.random() < 0.4:
                window, sinks = _log_int(rng, 16, 4096), rng.choice([0, 1, 4, 16])
        else:
            n = _log_int(rng, 1, 64)
            new_hi = _log_int(rng, 1, 250)
            past = (new_hi * page, new_hi * page * 2)
            new = (rng.randint(1, new_hi), new_hi)
        c = _case(op, n, past, new, heads, kv_heads, dim, page, dtype, form, window, sinks, rot, layout, axes, norm, branch)
        # no larger than the largest listed cases: cells, padded scores, and rows
        q, p = _lengths(c)
        cells = n * (max(p) + max(q)) * kv_heads * dim
        scores = n * heads * max(q) * (max(p) + max(q)) if branch else 0
        if cells <= 2.2e8 and scores <= 6e8 and (dtype != "f32" or scores <= 1e8) and sum(q) * (heads + 2 * kv_heads) * dim <= 2.8e8:
            return c


def _spread(lo, hi, n, step):
    """n lengths over lo .. hi by multiples of an irrational step; the first is hi."""
    return [hi - int((hi - lo + 1) * ((b * step) % 1.0)) for b in range(n)]


def _lengths(case):
    """(new tokens, tokens in the cache before them) of each sequence."""
    new = _spread(case["new_lo"], case["new_hi"], case["n_seqs"], 0.6180339887)
    past = _spread(case["past_lo"], case["past_hi"], case["n_seqs"], 0.7548776662)
    return new, past


def _trees(case):
    """Each sequence's parents and depths, by a fixed rule: the parent is one of the `branch` tokens
    before (now and then none: another continuation from the earlier tokens)."""
    out = []
    for b, n in enumerate(_lengths(case)[0]):
        rng = random.Random(1000 * case["branch"] + b)
        parents, depth = [], []
        for i in range(n):
            p = -1 if i == 0 or (case["branch"] > 1 and rng.random() < 0.05) else rng.randint(max(0, i - max(case["branch"], 1)), i - 1)
            parents.append(p)
            depth.append(0 if p < 0 else depth[p] + 1)
        out.append((parents, depth))
    return out


def _path(parents):
    """The last token and its ancestors, from the first on."""
    path, i = [], len(parents) - 1
    while i >= 0:
        path.append(i)
        i = parents[i]
    return path[::-1]


def _frequencies(case):
    """Radians per position of each pair, and the pair's axis (of three: one part in four of the pairs
    time, the rest height and width)."""
    half = case["rot"] // 2
    freq = [_BASE ** (-2.0 * i / case["rot"]) for i in range(half)]
    cut = {1: [], 2: [half // 2], 3: [half // 4, half // 4 + (half - half // 4) // 2]}[case["axes"]]
    return freq, [sum(i >= c for c in cut) for i in range(half)]


def _pow2(e):
    """2^e in fp32, for whole e from -126 to 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x):
    """Codes and scale bytes of rows of fp32 values: x ~ code * 2^(byte - 127), the least power of
    two that brings the row's largest value to 448 or below."""
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))      # m in [0.5, 1), value m * 2^e
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(-127, 127)
    e = torch.where(m == 0, torch.full_like(e, -127), e)
    half = torch.div(e, 2, rounding_mode="floor")           # 2^-e in two exact steps
    y = x * _pow2(-half) * _pow2(half - e)
    return y.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8).squeeze(-1)


def _values(codes, scale):
    """The fp32 values of codes with scale bytes."""
    if scale is None:
        return codes.float()
    e = scale.to(torch.int32).unsqueeze(-1) - 127
    half = torch.div(e, 2, rounding_mode="floor")
    return codes.float() * _pow2(half) * _pow2(e - half)


class State:
    pass


def _inputs(case, seed):
    s = State()
    s.case = case
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dt = _TYPES[case["dtype"]]
    h, hk, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    new, past = _lengths(case)
    fork = case["op"] == "fork"
    s.new, s.pos = ([0] * len(new) if fork else new), past
    s.kv = [a + b for a, b in zip(s.new, past)]
    total = sum(s.new)
    # the pages of a sequence lie anywhere in the pool
    need = [-(-k // page) for k in s.kv]
    n_pages = sum(need) + (sum(new) if fork else 0) + 3
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    s.table = torch.zeros(len(new), max(1, max(need)), dtype=torch.int32)
    at = 0
    s.src, s.dst = [], []
    for b, k in enumerate(need):
        s.table[b, :k] = order[at:at + k]
        at += k
        if fork:
            s.src += s.table[b, k - new[b]:k].tolist()
    if fork:
        s.dst = order[at:at + len(s.src)].tolist()
    s.n_pages = n_pages

    # keys with a few channels much larger than the rest, as projections of real text have them
    loud = 1.0 + 3.0 * (torch.arange(d, device=dev) % 16 == 3)

    def filled(gain):
        x = torch.randn(n_pages, hk, page, d, generator=gen, device=dev, dtype=dt)
        x *= gain
        if case["form"] == "same":
            return x, None
        return _quantise(x.float())

    (s.k_pool, s.k_scale), (s.v_pool, s.v_scale) = filled(loud.to(dt)), filled(1.0)
    # queries, keys and values of the new tokens are columns of one projection's output
    qkv = torch.randn(max(total, 1), h + 2 * hk, d, generator=gen, device=dev, dtype=dt)[:total]
    qkv[:, h:h + hk] *= loud.to(dt)
    s.q, s.k, s.v = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
    s.weights = (1.0 + 0.2 * torch.randn(2, d, generator=torch.Generator().manual_seed(seed))) if case["norm"] else None
    # positions along several axes are given by the caller: a patch's frame, row and column
    s.positions = None
    if case["axes"] > 1:
        s.positions = torch.randint(0, 300, (case["axes"], max(total, 1)), generator=gen, device=dev, dtype=torch.int32)[:, :total]
    s.trees = _trees(case) if case["branch"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2607_18582_gb300 import mure
        s.ctx = mure.mure_create(0)
        buffers = (s.k_pool, s.v_pool) if case["form"] == "same" else (s.k_pool, s.v_pool, s.k_scale, s.v_scale)
        s.cache = mure.mure_tokens_create(s.ctx, case["kv_heads"], case["dim"], case["page"], s.n_pages,
                                          dtype=case["dtype"], form=case["form"], buffers=buffers)
        s.parents = [p for parents, _ in s.trees for p in parents] if s.trees else None
        s.plan = mure.mure_tokens_plan(s.cache, case["heads"], s.new, s.pos, s.kv, s.table.numpy(),
                                       window=case["window"], sinks=case["sinks"], parents=s.parents)
        if case["op"] in ("rotate", "place", "step"):
            freq, axis = _frequencies(case)
            s.rotary = mure.mure_rotary_create(s.ctx, case["dim"], case["rot"], layout=case["layout"], freq=freq, axis=axis,
                                               n_axes=case["axes"], eps=_EPS,
                                               q_weight=s.weights[0].numpy() if case["norm"] else None,
                                               k_weight=s.weights[1].numpy() if case["norm"] else None)
        if case["op"] == "step":
            s.kept = [_path(parents) for parents, _ in s.trees]
        s.src, s.dst = np.array(s.src, np.int32), np.array(s.dst, np.int32)
        s.mure = mure
        return s
    # whose token each row is, and the cells, as indices for the plain form
    dev, new = s.q.device, torch.tensor(s.new)
    s.seq = torch.repeat_interleave(torch.arange(len(new)), new).to(dev)
    s.idx = (torch.arange(int(new.sum())) - torch.repeat_interleave(new.cumsum(0) - new, new)).to(dev)
    s.gpu_table, s.gpu_pos = s.table.long().to(dev), torch.tensor(s.pos, device=dev)
    s.gpu_kv = torch.tensor(s.kv, device=dev)
    s.gpu_src, s.gpu_dst = torch.tensor(s.src, device=dev), torch.tensor(s.dst, device=dev)
    most = max(max(s.new), 1)
    s.depth = s.idx
    if s.trees:
        # line[b, i, a]: token a of sequence b is i or one of its ancestors
        s.depth = torch.tensor([d for _, depth in s.trees for d in depth], device=dev)
        s.line = torch.zeros(len(s.new), most, most, dtype=torch.bool)
        s.far = torch.zeros(len(s.new), most, dtype=torch.int64)
        for b, (parents, depth) in enumerate(s.trees):
            s.far[b, :len(depth)] = torch.tensor(depth)
            for i, p in enumerate(parents):
                if p >= 0:
                    s.line[b, i] = s.line[b, p]
                s.line[b, i, i] = True
        s.line, s.far = s.line.to(dev), s.far.to(dev)
    if case["op"] == "step":
        kept = [_path(parents) for parents, _ in s.trees]
        s.keep_seq = torch.tensor([b for b, path in enumerate(kept) for _ in path], device=dev)
        s.keep_from = torch.tensor([i for path in kept for i in path], device=dev)
        s.keep_to = torch.tensor([i for path in kept for i in range(len(path))], device=dev)
    freq, axis = _frequencies(case)
    s.freq, s.axis = torch.tensor(freq, dtype=torch.float64, device=dev), torch.tensor(axis, dtype=torch.int64, device=dev)
    s.gpu_weights = s.weights.to(dev) if case["norm"] else None
    return s


def run(s):
    op = s.case["op"]
    if own:
        m = s.mure
        if op == "rotate":
            return m.mure_tokens_rotate(s.cache, s.plan, s.rotary, s.q, s.k, positions=s.positions)
        if op == "fork":
            m.mure_tokens_copy_pages(s.cache, s.src, s.dst)
            return s.k_pool, s.v_pool
        if op == "tree":
            return m.mure_tokens_attend(s.cache, s.plan, s.q, lse=True)
        q = m.mure_tokens_append_rotated(s.cache, s.plan, s.rotary, s.q, s.k, s.v, positions=s.positions)
        if op == "place":
            if s.case["form"] == "same":
                return q, s.k_pool, s.v_pool
            return (q, *m.mure_tokens_read(s.cache, s.plan, new=True))
        out, lse = m.mure_tokens_attend(s.cache, s.plan, q, lse=True)
        m.mure_tokens_keep(s.cache, s.plan, s.kept)
        return out, lse, s.k_pool, s.v_pool
    if op == "fork":
        s.k_pool[s.gpu_dst] = s.k_pool[s.gpu_src]
        s.v_pool[s.gpu_dst] = s.v_pool[s.gpu_src]
        return s.k_pool, s.v_pool
    if op == "tree":
        return _plain_attend(s, s.q)
    q, k = _plain_rotate(s, s.q, 0), _plain_rotate(s, s.k, 1)
    if op == "rotate":
        return q, k
    _plain_write(s, k, s.v)
    if op == "place":
        if s.case["form"] == "same":
            return q, s.k_pool, s.v_pool
        return (q, *_plain_read(s))
    out, lse = _plain_attend(s, q)
    page = s.case["page"]
    old, cell = s.gpu_pos[s.keep_seq] + s.keep_from, s.gpu_pos[s.keep_seq] + s.keep_to
    a, b = s.gpu_table[s.keep_seq, old // page], s.gpu_table[s.keep_seq, cell // page]
    s.k_pool[b, :, cell % page] = s.k_pool[a, :, old % page]
    s.v_pool[b, :, cell % page] = s.v_pool[a, :, old % page]
    return out, lse, s.k_pool, s.v_pool


def _plain_rotate(s, x, which):
    c = s.case
    half, d = c["rot"] // 2, c["dim"]
    y = x.float()
    if c["norm"]:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + _EPS) * s.gpu_weights[which]
    at = s.positions.double() if s.positions is not None else (s.gpu_pos[s.seq] + s.depth).double()[None]
    angle = at[s.axis].T * s.freq                          # [tokens][pairs], in 64 bits
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if c["layout"] == "halves":
        a, b = y[..., :half], y[..., half:2 * half]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = y[..., :2 * half:2], y[..., 1:2 * half:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((turned, y[..., 2 * half:d]), -1).to(x.dtype)


def _plain_write(s, k, v):
    page = s.case["page"]
    cell = s.gpu_pos[s.seq] + s.idx
    at = s.gpu_table[s.seq, cell // page]
    if s.k_scale is None:
        s.k_pool[at, :, cell % page] = k
        s.v_pool[at, :, cell % page] = v
        return
    (kc, ke), (vc, ve) = _quantise(k.float()), _quantise(v.float())
    s.k_pool.view(torch.uint8)[at, :, cell % page] = kc.view(torch.uint8)
    s.v_pool.view(torch.uint8)[at, :, cell % page] = vc.view(torch.uint8)
    s.k_scale[at, :, cell % page] = ke
    s.v_scale[at, :, cell % page] = ve


def _plain_read(s):
    page, dt = s.case["page"], _TYPES[s.case["dtype"]]
    cell = s.gpu_pos[s.seq] + s.idx
    at = s.gpu_table[s.seq, cell // page]

    def rows(pool, scale):
        return _values(pool.view(torch.uint8)[at, :, cell % page].view(torch.float8_e4m3fn), scale[at, :, cell % page]).to(dt)

    return rows(s.k_pool, s.k_scale), rows(s.v_pool, s.v_scale)


def _plain_attend(s, q_rows):
    c = s.case
    h, hk, d, g = c["heads"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"]
    dev, n, most = s.q.device, len(s.new), max(max(s.new), 1)

    def cells(pool, scale):
        x = pool.view(torch.uint8)[s.gpu_table].view(pool.dtype) if scale is not None else pool[s.gpu_table]
        x = _values(x, None if scale is None else scale[s.gpu_table])
        return x.transpose(1, 2).reshape(n, hk, -1, d)       # [n][hk][cells][d]

    k, v = cells(s.k_pool, s.k_scale), cells(s.v_pool, s.v_scale)
    q = torch.zeros(n, most, h, d, device=dev)
    q[s.seq, s.idx] = q_rows.float()
    q = q.view(n, most, hk, g, d).permute(0, 2, 3, 1, 4).reshape(n, hk, g * most, d)
    scores = torch.matmul(q, k.transpose(-1, -2)).view(n, hk, g, most, -1) * d ** -0.5
    # a cell's position and whether it is one of the tree's
    cell = torch.arange(k.shape[2], device=dev)
    node = cell[None] - s.gpu_pos[:, None]                                    # [n][cells]
    inside = (node >= 0) & (node < most)
    row = node.clamp(0, most - 1)
    at = torch.where(inside, s.gpu_pos[:, None] + s.far.gather(1, row), cell[None])
    mine = s.gpu_pos[:, None] + s.far                                         # [n][most] a row's position
    seen = torch.where(inside[:, None], s.line.gather(2, row[:, None].expand(n, most, -1)), (node < 0)[:, None])
    seen &= (cell[None] < s.gpu_kv[:, None])[:, None]
    if c["window"]:
        seen &= (at[:, None] > mine[..., None] - c["window"]) | (at < c["sinks"])[:, None]
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    scores.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    total = scores.sum(-1, keepdim=True)
    lse = (total.log() + top).squeeze(-1)
    out = torch.matmul(scores.view(n, hk, g * most, -1), v).view(n, hk, g, most, d) / total.masked_fill(total == 0, 1.0)
    out = out.permute(0, 3, 1, 2, 4).reshape(n, most, h, d)[s.seq, s.idx]
    lse = lse.permute(0, 3, 1, 2).reshape(n, most, h)[s.seq, s.idx]
    return out.to(_TYPES[c["dtype"]]), lse


def _visible(case):
    """Sum over the tree's tokens of the cells that each may attend to, and the cells of all sequences
    that any of their tokens may attend to."""
    pairs = cells = 0
    w, s = case["window"], case["sinks"]
    for (n, p), (parents, depth) in zip(zip(*_lengths(case)), _trees(case)):
        before = 0
        for i in range(n):
            at = p + depth[i]
            first = min(p, max(0, at - w + 1)) if w else 0
            past = p - first + min(s, first)
            # ancestors whose position the window or the first tokens hold
            mine = sum(1 for t in range(depth[i] + 1) if not w or t > depth[i] - w or p + t < s)
            pairs += past + mine
            before = max(before, past)
        cells += before + n
    return pairs, cells


def work(case):
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    b = _BYTES[case["dtype"]]
    cell = 2 * hk * (d * b if case["form"] == "same" else d + 1)     # keys and values of one token
    new, past = _lengths(case)
    n = sum(new)
    if case["op"] == "rotate":
        return {"bytes": 2 * n * (h + hk) * d * b, "flops": 8 * n * (h + hk) * d}
    if case["op"] == "fork":
        return {"bytes": 2 * n * case["page"] * cell, "flops": 0}
    place = {"bytes": n * ((2 * h + 2 * hk) * d * b + cell), "flops": 8 * n * (h + hk) * d}
    if case["op"] == "place":
        if case["form"] != "same":      # the cells are read back
            place["bytes"] += n * (cell + 2 * hk * d * b)
        return place
    pairs, cells = _visible(case)
    attend = {"bytes": cells * cell + n * h * (2 * d * b + 4), "flops": 4 * d * h * pairs}
    if case["op"] == "tree":
        return attend
    kept = sum(sum(i != k for k, i in enumerate(_path(parents))) for parents, _ in _trees(case))
    # (q as rotated is written and read between the two)
    return {"bytes": place["bytes"] + attend["bytes"] + 2 * kept * cell, "flops": place["flops"] + attend["flops"]}


def exact(case, seed):
    """The outputs in 64 bits, a sequence and a cached head at a time."""
    if case["op"] in ("tree", "step") and work(case)["flops"] > 4e12:
        return None
    s = _inputs(case, seed)
    page, hk, d, g = case["page"], case["kv_heads"], case["dim"], case["heads"] // case["kv_heads"]
    rows_of = [sum(s.new[:b]) for b in range(len(s.new) + 1)]

    def power(e):
        return ((e.long() + 1023) << 52).view(torch.float64)

    def wide(codes, scale):
        x = codes.double()
        return x if scale is None else x * power(scale.long() - 127)[..., None]

    def turned(x, which):
        """Each pair as a complex number, multiplied by exp(i angle)."""
        y = x.double()
        if case["norm"]:
            y = y / torch.sqrt(torch.mean(y ** 2, -1, keepdim=True) + _EPS) * s.weights[which].double().to(y.device)
        if s.positions is None:
            at = [s.pos[b] + (s.trees[b][1][i] if s.trees else i) for b in range(len(s.new)) for i in range(s.new[b])]
            where = torch.tensor([at], dtype=torch.float64, device=y.device)
        else:
            where = s.positions.double()
        freq, axis = _frequencies(case)
        half, out = case["rot"] // 2, y.clone()
        for i in range(half):
            one, two = (i, i + half) if case["layout"] == "halves" else (2 * i, 2 * i + 1)
            turn = torch.polar(torch.ones_like(where[axis[i]]), where[axis[i]] * freq[i])[:, None]
            z = torch.complex(y[..., one], y[..., two]) * turn
            out[..., one], out[..., two] = z.real, z.imag
        return out

    if case["op"] == "fork":
        k, v = s.k_pool.double(), s.v_pool.double()
        for a, b in zip(s.src, s.dst):
            k[b], v[b] = k[a].clone(), v[a].clone()
        return k, v
    if case["op"] != "tree":
        q, k = turned(s.q, 0), turned(s.k, 1)
        if case["op"] == "rotate":
            return q, k
        if case["op"] == "step":
            # what attention reads are rows in the activations' type
            q, k = (x.to(_TYPES[case["dtype"]]).double() for x in (q, k))
    if case["op"] == "place" and case["form"] != "same":
        def stored(x):
            # the cells hold codes of the rows in the activations' type
            x = x.to(_TYPES[case["dtype"]]).double()
            most = x.abs().amax(-1, keepdim=True)
            e = torch.ceil(torch.log2(most / 448.0))
            e = torch.where(most * power(-e) > 448.0, e + 1, e)
            e = torch.where(most * power(1 - e) <= 448.0, e - 1, e).clamp(-127, 127)
            y = x * power(-e)
            # three bits after the leading one, down to 2^-9; ties to even
            step = power(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
            return torch.round(y / step) * step * power(e)
        return q, stored(k), stored(s.v)

    k_pool, v_pool = wide(s.k_pool, s.k_scale), wide(s.v_pool, s.v_scale)

    def put(pool, b, cell, row):
        pool[int(s.table[b, cell // page]), :, cell % page] = row

    def take(pool, b, cell):
        return pool[int(s.table[b, cell // page]), :, cell % page].clone()

    if case["op"] in ("place", "step"):
        for b, n in enumerate(s.new):
            cell = torch.arange(s.pos[b], s.pos[b] + n)
            ids = s.table[b, cell // page].long().to(k_pool.device)
            cell = cell.to(k_pool.device)
            k_pool[ids, :, cell % page] = k[rows_of[b]:rows_of[b + 1]]
            v_pool[ids, :, cell % page] = s.v[rows_of[b]:rows_of[b + 1]].double()
        if case["op"] == "place":
            return q, k_pool, v_pool
    else:
        q = s.q.double()

    outs, lses = [], []
    for b, n in enumerate(s.new):
        ids = s.table[b, :-(-s.kv[b] // page)].long().to(k_pool.device)
        kb = k_pool[ids].transpose(1, 2).reshape(-1, hk, d)[:s.kv[b]]
        vb = v_pool[ids].transpose(1, 2).reshape(-1, hk, d)[:s.kv[b]]
        parents, depth = s.trees[b]
        at = torch.cat((torch.arange(s.pos[b]), s.pos[b] + torch.tensor(depth, dtype=torch.int64)))
        seen = torch.zeros(n, s.kv[b], dtype=torch.bool)
        seen[:, :s.pos[b]] = True
        for i in range(n):
            a = i
            while a >= 0:
                seen[i, s.pos[b] + a] = True
                a = parents[a]
        if case["window"]:
            mine = s.pos[b] + torch.tensor(depth)[:, None]
            seen &= (mine - at[None] < case["window"]) | (at[None] < case["sinks"])
        seen = seen.to(k_pool.device)
        out = torch.empty(n, hk * g, d, dtype=torch.float64, device=k_pool.device)
        lse = torch.empty(n, hk * g, dtype=torch.float64, device=k_pool.device)
        for j in range(hk * g):
            z = q[rows_of[b]:rows_of[b + 1], j] @ kb[:, j // g].T / math.sqrt(d)
            z = z.masked_fill(~seen, -math.inf)
            lse[:, j] = torch.logsumexp(z, -1)
            out[:, j] = torch.softmax(z, -1) @ vb[:, j // g]
        outs.append(out)
        lses.append(lse)
    if case["op"] == "tree":
        return torch.cat(outs), torch.cat(lses)
    for b in range(len(s.new)):
        for to, i in enumerate(_path(s.trees[b][0])):
            for pool in (k_pool, v_pool):
                put(pool, b, s.pos[b] + to, take(pool, b, s.pos[b] + i))
    return torch.cat(outs), torch.cat(lses), k_pool, v_pool
