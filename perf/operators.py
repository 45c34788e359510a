"""The operators of a paged token cache as cases that can be timed and checked.

A network that attends over a sequence keeps the keys and values of its earlier tokens: the
memo table of a sequence model, shared by every mutant that leaves the layers before it alone.
Three operators deal with it:

  write   new tokens' keys and values go into the cells of their sequences' pages, as they are
          or as e4m3 codes with one power-of-two scale per token and head, and are read back
          (what a layer stores is what its later readers see);
  read    whole sequences are gathered from their pages into dense rows;
  attend  queries of a chunk of new tokens (one token each in a decoding step) attend over the
          cells of their sequences, causally, optionally within a sliding window plus the first
          few tokens.  The output and the log of each row's softmax sum come back.

Fields of a case: `op`; `n_seqs` sequences with `past_lo` .. `past_hi` tokens in the cache and
`new_lo` .. `new_hi` new ones (both spread over the sequences by a fixed rule); `heads` query
heads on `kv_heads` cached ones, of `dim` values; `page` cells per page; `dtype` of the
activations; `form` of the cells ("same" as the activations, or "e4m3"); `window` (0: none)
and `sinks`.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _case(op, n_seqs, past, new, heads, kv_heads, dim, page, dtype, form, window=0, sinks=0):
    return {"op": op, "n_seqs": n_seqs, "past_lo": past[0], "past_hi": past[1], "new_lo": new[0], "new_hi": new[1],
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype, "form": form,
            "window": window, "sinks": sinks}


def listed():
    def named(name, *a, **k):
        return dict(_case(*a, **k), name=name)

    return [
        # one decoding step of a small batch: a token per sequence, launches count
        named("write_token_e4m3", "write", 48, (100, 4000), (1, 1), 32, 8, 128, 16, "bf16", "e4m3"),
        # the prompts of a test set entering the cache
        named("write_prompts_e4m3", "write", 24, (0, 0), (500, 4100), 32, 8, 128, 16, "bf16", "e4m3"),
        # a quantised cache read back for a layer that wants dense rows
        named("read_e4m3", "read", 16, (900, 20000), (0, 0), 32, 8, 128, 16, "bf16", "e4m3"),
        # odd head counts and lengths, heads of 80 values
        named("read_odd", "read", 7, (1, 3001), (0, 0), 15, 5, 80, 32, "f16", "same"),
        # one sequence, one token: the latency of a single answer
        named("token_one", "attend", 1, (700, 700), (1, 1), 32, 8, 128, 16, "bf16", "same"),
        # a decoding step of many sequences of very different lengths on a quantised cache
        named("token_batch_e4m3", "attend", 64, (500, 12000), (1, 1), 32, 8, 128, 16, "bf16", "e4m3"),
        # two long documents: few rows, a long axis
        named("token_long", "attend", 2, (100001, 131071), (1, 1), 32, 8, 128, 64, "bf16", "same"),
        # a decoding step within a window and the first tokens
        named("token_window", "attend", 96, (300, 9000), (1, 1), 24, 4, 64, 16, "f16", "same", window=1024, sinks=4),
        # prompts that continue earlier ones, ragged
        named("chunk_ragged", "attend", 12, (0, 6000), (90, 700), 32, 8, 128, 16, "bf16", "same"),
        # chunks within a window and the first tokens, on a quantised cache
        named("chunk_window_e4m3", "attend", 3, (4000, 9000), (1500, 2500), 16, 2, 64, 32, "bf16", "e4m3", window=1024,
              sinks=4),
        # a long chunk in the middle of a long document, the largest work here
        named("chunk_long", "attend", 1, (8192, 8192), (8192, 8192), 32, 8, 128, 64, "bf16", "same"),
        # the fp32 activations of this framework's own networks
        named("chunk_f32", "attend", 6, (0, 1500), (33, 400), 12, 4, 64, 16, "f32", "same"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    while True:
        op = rng.choice(["write", "read", "attend", "attend", "attend"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        form = rng.choice(["same", "e4m3"])
        kv_heads = rng.choice([1, 2, 3, 4, 5, 8])
        heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 6, 8])
        dim = rng.choice([32, 40, 64, 64, 80, 96, 128, 128, 128])
        page = rng.choice([8, 16, 16, 32, 64, 128])
        window, sinks = 0, 0
        if op == "write":
            n = _log_int(rng, 1, 200)
            new_hi = 1 if rng.random() < 0.4 else _log_int(rng, 2, 4100)
            new = (max(1, new_hi // rng.choice([1, 3, 20])), new_hi)
            past_hi = _log_int(rng, 1, 4000)
            past = (rng.randint(0, past_hi), past_hi)
        elif op == "read":
            n = _log_int(rng, 1, 60)
            past_hi = _log_int(rng, 10, 20000)
            past, new = (rng.randint(0, past_hi), past_hi), (0, 0)
        else:
            if rng.random() < 0.5:   # a decoding step
                n = _log_int(rng, 1, 100)
                past_hi = _log_int(rng, 20, 100000)
                past, new = (rng.randint(0, past_hi), past_hi), (1, 1)
            else:
                n = _log_int(rng, 1, 16)
                new_hi = _log_int(rng, 2, 6000)
                past_hi = _log_int(rng, 10, 12000)
                past, new = (rng.randint(0, past_hi), past_hi), (rng.randint(1, new_hi), new_hi)
            if rng.random() < 0.4:
                window, sinks = _log_int(rng, 16, 4096), rng.choice([0, 1, 4, 16])
        c = _case(op, n, past, new, heads, kv_heads, dim, page, dtype, form, window, sinks)
        # no larger than the largest listed case: the cells of a sequence's padded length, the
        # scores of padded rows, and the rows themselves
        q, p = _lengths(c)
        kv = max(a + b for a, b in zip(q, p))
        cells, scores = n * kv * kv_heads * dim, n * heads * max(q) * kv
        if cells <= 2.5e8 and scores <= 1.5e9 and (dtype != "f32" or scores <= 2e8) and n * max(q) * heads * dim <= 3e7 * (10 if op == "write" else 1):
            return c


def _spread(lo, hi, n, step):
    """n lengths over lo .. hi by multiples of an irrational step; the first is hi."""
    return [hi - int((hi - lo + 1) * ((b * step) % 1.0)) for b in range(n)]


def _lengths(case):
    """(new tokens, tokens in the cache before them) of each sequence."""
    new = _spread(case["new_lo"], case["new_hi"], case["n_seqs"], 0.6180339887)
    past = _spread(case["past_lo"], case["past_hi"], case["n_seqs"], 0.7548776662)
    return new, past


def _visible(case):
    """Sum over the query tokens of the cells that each may attend to, and the cells of all
    sequences that any of their query tokens may attend to."""
    pairs = cells = 0
    w, s = case["window"], case["sinks"]
    for q, p in zip(*_lengths(case)):
        if q == 0:
            continue
        if w == 0:
            pairs += q * p + q * (q + 1) // 2
            cells += p + q
        else:
            for i in (range(p, p + q)):
                first = max(0, i - w + 1)
                pairs += i + 1 - first + min(s, first)
            first = max(0, p - w + 1)
            cells += p + q - first + min(s, first)
    return pairs, cells


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
    s.new, s.pos = new, past
    s.kv = [a + b for a, b in zip(new, past)]
    total = sum(new)
    # the pages of a sequence lie anywhere in the pool
    rows = max(1, -(-max(s.kv) // page))
    need = [-(-k // page) for k in s.kv]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    s.table = torch.zeros(len(new), rows, dtype=torch.int32)
    at = 0
    for b, k in enumerate(need):
        s.table[b, :k] = order[at:at + k]
        at += k

    # keys with a few channels much larger than the rest, as projections of real text have them
    loud = 1.0 + 3.0 * (torch.arange(d, device=dev) % 16 == 3)

    def filled(gain):
        x = torch.randn(n_pages, hk, page, d, generator=gen, device=dev, dtype=torch.float32 if dt == torch.float32 else dt)
        x *= gain
        if case["form"] == "same":
            return x, None
        return _quantise(x.float())

    (s.k_pool, s.k_scale), (s.v_pool, s.v_scale) = filled(loud.to(dt)), filled(1.0)
    # queries, keys and values of the new tokens are columns of one projection's output
    qkv = torch.randn(max(total, 1), h + 2 * hk, d, generator=gen, device=dev, dtype=dt)[:total]
    qkv[:, h:h + hk] *= loud.to(dt)
    s.q, s.k, s.v = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
    s.n_pages = n_pages
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2607_18582_gb300 import mure
        s.ctx = mure.mure_create(0)
        buffers = (s.k_pool, s.v_pool) if case["form"] == "same" else (s.k_pool, s.v_pool, s.k_scale, s.v_scale)
        s.cache = mure.mure_tokens_create(s.ctx, case["kv_heads"], case["dim"], case["page"], s.n_pages,
                                          dtype=case["dtype"], form=case["form"], buffers=buffers)
        s.plan = mure.mure_tokens_plan(s.cache, case["heads"], s.new, s.pos, s.kv, s.table.numpy(),
                                       window=case["window"], sinks=case["sinks"])
        s.mure = mure
        return s
    # whose token each row is, and the cells that are held, as indices for the plain form
    dev, new = s.q.device, torch.tensor(s.new)
    s.seq = torch.repeat_interleave(torch.arange(len(new)), new).to(dev)
    s.idx = (torch.arange(int(new.sum())) - torch.repeat_interleave(new.cumsum(0) - new, new)).to(dev)
    s.gpu_table, s.gpu_pos = s.table.long().to(dev), torch.tensor(s.pos, device=dev)
    s.gpu_kv = torch.tensor(s.kv, device=dev)
    s.held = (torch.arange(s.table.shape[1] * case["page"], device=dev)[None] < s.gpu_kv[:, None]).nonzero()
    return s


def run(s):
    op = s.case["op"]
    if own:
        if op == "write":
            s.mure.mure_tokens_append(s.cache, s.plan, s.k, s.v)
            return s.mure.mure_tokens_read(s.cache, s.plan, new=True)
        if op == "read":
            return s.mure.mure_tokens_read(s.cache, s.plan)
        return s.mure.mure_tokens_attend(s.cache, s.plan, s.q, lse=True)
    if op == "write":
        return _plain_write(s)
    if op == "read":
        return _plain_read(s, s.held[:, 0], s.held[:, 1])
    return _plain_attend(s)


def _plain_write(s):
    page = s.case["page"]
    cell = s.gpu_pos[s.seq] + s.idx
    at = s.gpu_table[s.seq, cell // page]
    for x, pool, scale in ((s.k, s.k_pool, s.k_scale), (s.v, s.v_pool, s.v_scale)):
        if scale is None:
            pool[at, :, cell % page] = x
        else:
            codes, e = _quantise(x.float())
            pool.view(torch.uint8)[at, :, cell % page] = codes.view(torch.uint8)
            scale[at, :, cell % page] = e
    return _plain_read(s, s.seq, cell)


def _plain_read(s, seq, cell):
    page, dt = s.case["page"], _TYPES[s.case["dtype"]]
    at = s.gpu_table[seq, cell // page]

    def rows(pool, scale):
        if scale is None:
            return pool[at, :, cell % page]
        return _values(pool.view(torch.uint8)[at, :, cell % page].view(torch.float8_e4m3fn), scale[at, :, cell % page]).to(dt)

    return rows(s.k_pool, s.k_scale), rows(s.v_pool, s.v_scale)


def _plain_attend(s):
    c = s.case
    h, hk, d, g = c["heads"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"]
    dev, n, most = s.q.device, len(s.new), max(max(s.new), 1)

    def cells(pool, scale):
        x = pool.view(torch.uint8)[s.gpu_table].view(pool.dtype) if scale is not None else pool[s.gpu_table]
        x = _values(x, None if scale is None else scale[s.gpu_table])
        return x.transpose(1, 2).reshape(n, hk, -1, d)       # [n][hk][cells][d]

    k, v = cells(s.k_pool, s.k_scale), cells(s.v_pool, s.v_scale)
    q = torch.zeros(n, most, h, d, device=dev)
    q[s.seq, s.idx] = s.q.float()
    q = q.view(n, most, hk, g, d).permute(0, 2, 3, 1, 4).reshape(n, hk, g * most, d)
    scores = torch.matmul(q, k.transpose(-1, -2)).view(n, hk, g, most, -1) * d ** -0.5
    at = s.gpu_pos[:, None] + torch.arange(most, device=dev)                 # a row's position
    cell = torch.arange(k.shape[2], device=dev)
    seen = (cell <= at[..., None]) & (cell < s.gpu_kv[:, None, None])
    if c["window"]:
        seen &= (cell > at[..., None] - c["window"]) | (cell < c["sinks"])
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    scores.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    total = scores.sum(-1, keepdim=True)
    lse = (total.log() + top).squeeze(-1)
    out = torch.matmul(scores.view(n, hk, g * most, -1), v).view(n, hk, g, most, d) / total.masked_fill(total == 0, 1.0)
    out = out.permute(0, 3, 1, 2, 4).reshape(n, most, h, d)[s.seq, s.idx]
    lse = lse.permute(0, 3, 1, 2).reshape(n, most, h)[s.seq, s.idx]
    return out.to(_TYPES[c["dtype"]]), lse


def work(case):
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    b = _BYTES[case["dtype"]]
    cell = 2 * hk * (d * b if case["form"] == "same" else d + 1)     # keys and values of one token
    new, past = _lengths(case)
    if case["op"] == "write":    # new rows in, cells out; cells in, rows out
        return {"bytes": sum(new) * 2 * (2 * hk * d * b + cell), "flops": 0}
    if case["op"] == "read":
        return {"bytes": (sum(new) + sum(past)) * (2 * hk * d * b + cell), "flops": 0}
    pairs, cells = _visible(case)
    return {"bytes": cells * cell + sum(new) * h * (2 * d * b + 4), "flops": 4 * d * h * pairs}


def exact(case, seed):
    """The outputs in 64 bits, a sequence and a cached head at a time."""
    if case["op"] == "attend" and work(case)["flops"] > 4e12:
        return None
    s = _inputs(case, seed)
    page, hk, d, g = case["page"], case["kv_heads"], case["dim"], case["heads"] // case["kv_heads"]

    def power(e):
        return ((e.long() + 1023) << 52).view(torch.float64)

    def wide(codes, scale):
        x = codes.double()
        return x if scale is None else x * power(scale.long() - 127)[..., None]

    def cells(b, pool, scale, length):     # [length][hk][d]
        ids = s.table[b, :-(-length // page)].long().to(pool.device)
        x = pool.view(torch.uint8)[ids].view(pool.dtype) if scale is not None else pool[ids]
        x = wide(x, None if scale is None else scale[ids])
        return x.transpose(1, 2).reshape(-1, hk, d)[:length]

    if case["op"] == "read":
        out = [[cells(b, pool, scale, n) for b, n in enumerate(s.kv)]
               for pool, scale in ((s.k_pool, s.k_scale), (s.v_pool, s.v_scale))]
        return torch.cat(out[0]), torch.cat(out[1])
    if case["op"] == "write":
        def stored(x):
            if case["form"] == "same":
                return x.double()
            x = x.double()
            most = x.abs().amax(-1, keepdim=True)
            e = torch.ceil(torch.log2(most / 448.0))
            e = torch.where(most * power(-e) > 448.0, e + 1, e)
            e = torch.where(most * power(1 - e) <= 448.0, e - 1, e).clamp(-127, 127)
            y = x * power(-e)
            # three bits after the leading one, down to 2^-9; ties to even
            step = power(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
            return torch.round(y / step) * step * power(e)
        return stored(s.k), stored(s.v)

    outs, lses, row = [], [], 0
    for b, n in enumerate(s.new):
        if n == 0:
            continue
        k, v = cells(b, s.k_pool, s.k_scale, s.kv[b]), cells(b, s.v_pool, s.v_scale, s.kv[b])
        at = torch.arange(s.pos[b], s.pos[b] + n, device=k.device)[:, None]
        cell = torch.arange(s.kv[b], device=k.device)[None]
        hidden = cell > at
        if case["window"]:
            hidden = hidden | ((at - cell >= case["window"]) & (cell >= case["sinks"]))
        out = torch.empty(n, hk * g, d, dtype=torch.float64, device=k.device)
        lse = torch.empty(n, hk * g, dtype=torch.float64, device=k.device)
        for j in range(hk * g):
            z = s.q[row:row + n, j].double() @ k[:, j // g].T / math.sqrt(d)
            z = z.masked_fill(hidden, -math.inf)
            lse[:, j] = torch.logsumexp(z, -1)
            out[:, j] = torch.softmax(z, -1) @ v[:, j // g]
        outs.append(out)
        lses.append(lse)
        row += n
    if not outs:
        return torch.empty(0, hk * g, d, dtype=torch.float64), torch.empty(0, hk * g, dtype=torch.float64)
    return torch.cat(outs), torch.cat(lses)
