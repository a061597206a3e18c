"""Workloads of windowed attention and of the 4-bit cache, for timing and for checks.

Two operators of the cache, alone and together:

* attention with a sliding window and sinks: a query at position p sees the
  positions j <= p with j < sinks or j > p - window, in a decode step
  (``Cache.attention(q, window=, sinks=)``) and for the new tokens of a joined
  sequence (``Cache.prefill(id, q, window=, sinks=)``);
* a cache held in 4 bits (``Cache(..., kv_bits=4)``): a row of d elements of one
  token and head is ``low + scale * code`` with codes 0..15, decode attention
  over it, and joins (``Cache.insert`` of the new rows, ``Cache.prefill``).

``run`` computes them with elementary torch operations in 32 bits, or, where
``own`` is true, through the cache. K, V and q are N(0, 1) draws and token ids
are uniform in [0, 32000), as in ``workloads``.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

VOCAB = 32000
DTYPES = {"fp16": torch.float16, "fp32": torch.float32, "kv4": torch.float16}
# most K/V, q and o bytes and most FLOPs of a drawn case: no more than the
# largest listed decode call and prefill take
MOST_BYTES = 5.3e8
MOST_FLOPS = 1.3e11


def _decode(name, kv, rows, prompt, unique, heads=32, dim=128, chunk=64, branches=1, branch=0,
            unique_min=None, ordered=False, window=0, sinks=0):
    c = dict(kind="decode", kv=kv, rows=rows, prompt=prompt, branches=branches, branch=branch,
             unique_min=unique if unique_min is None else unique_min, unique_max=unique, heads=heads,
             dim=dim, chunk=chunk, ordered=ordered, window=window, sinks=sinks)
    return dict(c, name=name) if name else c


def _prefill(name, kind, kv, prefix, new, heads=32, dim=128, chunk=64, window=0, sinks=0):
    c = dict(kind=kind, kv=kv, prefix=prefix, new=new, heads=heads, dim=dim, chunk=chunk, window=window,
             sinks=sinks)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a tiny model: four rows, two heads, chunks of 16 (latency only)
        _decode("kv4_decode_tiny", "kv4", 4, 128, 32, heads=2, dim=64, chunk=16),
        # the benchmark's batch: a shared system prompt and private suffixes
        _decode("kv4_decode_bench", "kv4", 32, 1024, 512),
        # one user with a long private context: nothing is shared, one row
        _decode("kv4_decode_long", "kv4", 1, 0, 32765),
        # a large serving batch of ragged rows in the batch's own row order
        _decode("kv4_decode_ragged", "kv4", 128, 2048, 1024, unique_min=64, ordered=True),
        # a windowed layer over the benchmark's batch: the window ends inside the prompt
        _decode("window_decode_bench", "fp16", 32, 1024, 512, window=1024, sinks=4),
        # long private contexts of which a windowed layer reads the end
        _decode("window_decode_long", "fp16", 16, 300, 7800, unique_min=5000, window=2048, sinks=4,
                ordered=True),
        # a tiny fp32 model with a window shorter than a chunk's worth of rows
        _decode("window_decode_fp32", "fp32", 6, 100, 75, heads=4, dim=64, chunk=16, window=50, sinks=1),
        # both: a ragged batch, windowed, over the 4-bit cache
        _decode("kv4_window_decode", "kv4", 64, 1500, 2500, unique_min=700, window=1024, sinks=16),
        # a new message behind a cached conversation joins a 4-bit cache: rows written, prefill
        _prefill("kv4_join", "join", "kv4", 1024, 512),
        # a short turn with odd lengths, windowed layer of a 4-bit cache
        _prefill("kv4_window_join_short", "join", "kv4", 1500, 37, window=512, sinks=4),
        # a long document behind a long cached prompt, windowed layer
        _prefill("window_prefill_long", "prefill", "fp16", 6144, 2048, window=4096, sinks=4),
        # a prompt of its own, odd sizes, d = 64, a short window
        _prefill("window_prefill_d64", "prefill", "fp16", 0, 1999, heads=16, dim=64, window=333, sinks=2),
    ]


def _log(rng, lo, hi):
    """A whole number, uniform over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    heads = rng.choice([1, 2, 3, 4, 8, 16, 32, 32, 32])
    dim = rng.choice([64, 128, 128])
    chunk = rng.choice([16, 32, 64, 64, 64, 100, 128])
    kv = rng.choice(["kv4", "kv4", "kv4", "fp16", "fp16", "fp32"])
    kind = rng.choice(["decode", "decode", "decode", "prefill", "prefill"])
    windowed = kv != "kv4" or rng.random() < 0.4
    window = _log(rng, 16, 8192) if windowed else 0
    sinks = rng.choice([0, 1, 4, 4, 16, rng.randint(1, 128)]) if windowed else 0
    if kind == "decode":
        rows = _log(rng, 1, 128)
        prompt = 0 if rng.random() < 0.15 else _log(rng, 16, 8192)
        unique = _log(rng, 1, 32768 if rows <= 4 else 4096)
        least = max(1, int(unique * rng.choice([1.0, 1.0, rng.uniform(0.05, 1.0)])))
        branches, branch = 1, 0
        if prompt and rows >= 8 and rng.random() < 0.3:
            branches, branch = rng.randint(2, 4), _log(rng, 16, 1024)
        c = _decode(None, kv, rows, prompt, unique, heads, dim, chunk, branches, branch, least,
                    rng.random() < 0.4, window, sinks)
        # stored rows (also those outside the window) bound the inputs' size
        while work(c)["bytes"] > MOST_BYTES or work(dict(c, window=0))["bytes"] > 2 * MOST_BYTES:
            c["unique_max"] = c["unique_max"] * 2 // 3
            c["unique_min"] = min(c["unique_min"], c["unique_max"])
            c["prompt"] = max(16, c["prompt"] * 2 // 3) if c["prompt"] else 0
        return c
    if kv == "fp32":
        kv = "fp16"
    c = _prefill(None, "join" if kv == "kv4" else "prefill", kv, 0 if rng.random() < 0.2 else _log(rng, 16, 8192),
                 _log(rng, 1, 4096), heads, dim, chunk, window, sinks)
    while work(c)["flops"] > MOST_FLOPS:
        c["new"] = max(1, c["new"] * 2 // 3)
    return c


# -- sizes -------------------------------------------------------------------


def _spread(n, lo, hi):
    """n lengths spread evenly over [lo, hi] in a mixed order (a Weyl sequence)."""
    return [lo + int((hi - lo + 1) * ((i + 1) * 0.6180339887498949 % 1.0)) for i in range(n)]


def _unique_lens(case):
    return _spread(case["rows"], case["unique_min"], case["unique_max"])


def _row_bytes(case):
    """Bytes of one stored token's K and V over all heads."""
    d = case["dim"]
    return 2 * case["heads"] * {"fp16": 2 * d, "fp32": 4 * d, "kv4": d // 2 + 4}[case["kv"]]


def _io_bytes(case):
    """Bytes of one row of q and one of o."""
    return 2 * case["heads"] * case["dim"] * (4 if case["kv"] == "fp32" else 2)


def _visible(length, window, sinks):
    """Positions that the last of `length` tokens sees, as disjoint ranges."""
    lo = max(0, length - window) if window else 0
    return [(0, min(sinks, lo)), (lo, length)]


def _covered(ranges):
    """Number of integers in a union of half-open ranges."""
    n = end = 0
    for a, b in sorted(ranges):
        a = max(a, end)
        if b > a:
            n += b - a
            end = b
    return n


def work(case):
    """What a pass cannot do without: every stored token that some query sees
    read once (K and V, shared ones once for all rows), q in, o out, a join's
    new K/V rows in and their stored form out; 4 FLOPs per (query, visible
    token, head, dim)."""
    w, s, rb = case["window"], case["sinks"], _row_bytes(case)
    fl = 4 * case["heads"] * case["dim"]
    if case["kind"] == "decode":
        p, br = case["prompt"], case["branch"]
        segs, pairs = {}, 0
        for i, u in enumerate(_unique_lens(case)):
            for a, b in _visible(p + br + u, w, s):
                pairs += max(0, b - a)
                for key, x, y in (("p", 0, p), (i % case["branches"], p, p + br), (("u", i), p + br, p + br + u)):
                    segs.setdefault(key, []).append((max(a, x), min(b, y)))
        stored = sum(_covered([r for r in v if r[1] > r[0]]) for v in segs.values())
        return {"bytes": rb * stored + _io_bytes(case) * case["rows"], "flops": fl * pairs}
    L, n = case["prefix"] + case["new"], case["new"]
    pairs = sum(_covered(_visible(t, w, s)) for t in range(L - n + 1, L + 1))
    first = max(0, L - n + 1 - w) if w else 0
    bytes_ = rb * _covered([(0, min(s, first)), (first, L)]) + _io_bytes(case) * n
    if case["kind"] == "join":
        bytes_ += n * (_io_bytes(case) + rb)
    return {"bytes": bytes_, "flops": fl * pairs}


# -- inputs ------------------------------------------------------------------


def _draws(case, seed):
    """Token ids from a host generator, K/V/q rows from a GPU generator, both
    made from the seed alone; the order of the calls fixes the values."""
    ids = np.random.Generator(np.random.PCG64(seed))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DTYPES[case["kv"]]

    def rows(n):
        return torch.randn((n, case["heads"], case["dim"]), generator=gen, dtype=dt, device="cuda")

    def segment(n, first=None):
        t = ids.integers(0, VOCAB, n).astype(np.int32)
        if first is not None and n:
            t[0] = first
        return t, rows(n), rows(n)

    return ids, rows, segment


def _decode_inputs(case, seed):
    """The segments (tokens, K, V), per row the indices of its path's segments,
    and q by row. Rows are listed in the batch's order."""
    ids, rows, segment = _draws(case, seed)
    n, nb = case["rows"], case["branches"]
    segs = [segment(case["prompt"])]
    firsts = ids.permutation(VOCAB)[: n + nb]
    segs += [segment(case["branch"], firsts[n + b]) for b in range(nb)]
    segs += [segment(u, firsts[i]) for i, u in enumerate(_unique_lens(case))]
    paths = [[0, 1 + i % nb, 1 + nb + i] for i in range(n)]
    q = rows(n)
    if not case["ordered"]:
        # tree order: by the first token that differs from the other rows'
        key = [tuple(int(segs[j][0][0]) for j in p[1:] if len(segs[j][0])) for p in paths]
        order = sorted(range(n), key=lambda i: key[i])
        paths = [paths[i] for i in order]
    return segs, [[j for j in p if len(segs[j][0])] for p in paths], q


def _join_inputs(case, seed):
    """The cached conversation (prefix plus a tail of its own), the joining
    sequence (prefix plus new tokens), and the new tokens' q."""
    ids, rows, segment = _draws(case, seed)
    firsts = ids.permutation(VOCAB)[:2]
    prefix = segment(case["prefix"])
    tail = segment(40, firsts[0])
    new = segment(case["new"], firsts[1])
    return _cat([prefix, tail]), _cat([prefix, new]), rows(case["new"])


def _cat(segs):
    return (np.concatenate([s[0] for s in segs]), torch.cat([s[1] for s in segs]),
            torch.cat([s[2] for s in segs]))


# -- the 4-bit form, plain -----------------------------------------------------


def _codes(x):
    """Codes, scale and low of the rows x [n, H, d]."""
    low = x.amin(-1, keepdim=True).float()
    scale = ((x.amax(-1, keepdim=True).float() - low) / 15).half().float()
    # the quotient decides between neighbouring codes: in 64 bits
    c = torch.round((x.double() - low.double()) / scale.double()).clamp_(0, 15)
    c = torch.where(scale > 0, c, torch.zeros_like(c))
    return c.to(torch.uint8), scale, low


def _values(codes):
    c, scale, low = codes
    return c.float() * scale + low


def _stored(case, k, v):
    """K and V as the plain program's cache keeps them."""
    return (_codes(k), _codes(v)) if case["kv"] == "kv4" else (k, v)


def _rows32(case, stored):
    return tuple(_values(t) if case["kv"] == "kv4" else t.float() for t in stored)


# -- passes ------------------------------------------------------------------


def _cache(case, lens):
    from paper_2402_15220_amd.cache import Cache

    slots = sum(-(-n // case["chunk"]) + 2 for n in lens) + 8
    return Cache(case["chunk"], case["heads"], case["dim"], slots, dtype=DTYPES[case["kv"]],
                 kv_bits=4 if case["kv"] == "kv4" else None)


def _window(case):
    return {"window": case["window"], "sinks": case["sinks"]} if case["window"] else {}


def prepare(case, seed):
    if case["kind"] == "decode":
        segs, paths, q = _decode_inputs(case, seed)
        state = {"case": case, "own": own, "q": q}
        if not own:
            state["paths"] = paths
            state["segs"] = [_stored(case, s[1], s[2]) if len(s[0]) else None for s in segs]
            return state
        cache = _cache(case, [len(s[0]) for s in segs])
        for i, p in enumerate(paths):
            cache.insert(i, *_cat([segs[j] for j in p]))
        cache.prepare(**_window(case))
        state["cache"] = cache
        state["ids"] = np.arange(len(paths), dtype=np.int64) if case["ordered"] else None
        return state
    old, new, q = _join_inputs(case, seed)
    p = case["prefix"]
    state = {"case": case, "own": own, "q": q, "new": new}
    if own:
        cache = _cache(case, [p, 40, case["new"]])
        cache.insert(0, *old)
        if case["kind"] == "prefill":
            cache.insert(1, *new)
        state["cache"] = cache
    else:
        cached = p if case["kind"] == "join" else p + case["new"]
        state["cached"] = _stored(case, new[1][:cached], new[2][:cached])
    return state


def _plain_decode(state):
    case, q = state["case"], state["q"]
    segs = [None if s is None else _rows32(case, s) for s in state["segs"]]
    out = torch.empty_like(q)
    for r, path in enumerate(state["paths"]):
        k = torch.cat([segs[j][0] for j in path])
        v = torch.cat([segs[j][1] for j in path])
        L = k.shape[0]
        if case["window"] and L > case["window"]:
            lo = L - case["window"]
            s = min(case["sinks"], lo)
            k, v = torch.cat([k[:s], k[lo:]]), torch.cat([v[:s], v[lo:]])
        s = (k * q[r].float()).sum(-1) / math.sqrt(case["dim"])
        e = torch.exp(s - s.amax(0))
        out[r] = ((e.unsqueeze(-1) * v).sum(0) / e.sum(0).unsqueeze(-1)).to(out.dtype)
    return out


def _plain_prefill(state):
    case, q = state["case"], state["q"]
    k, v = _rows32(case, state["cached"])
    if case["kind"] == "join":
        p = case["prefix"]
        kn, vn = _rows32(case, _stored(case, state["new"][1][p:], state["new"][2][p:]))
        k, v = torch.cat([k, kn]), torch.cat([v, vn])
    L, n, w = k.shape[0], q.shape[0], case["window"]
    kt = k.permute(1, 2, 0).contiguous()
    vh = v.transpose(0, 1).contiguous()
    qh = q.float().transpose(0, 1).contiguous()
    out = torch.empty_like(q)
    j = torch.arange(L, device=q.device)
    step = max(1, (1 << 28) // (L * q.shape[1]))
    for i in range(0, n, step):
        pos = (L - n + i + torch.arange(min(step, n - i), device=q.device)).unsqueeze(1)
        seen = j <= pos
        if w:
            seen &= (j > pos - w) | (j < case["sinks"])
        s = torch.matmul(qh[:, i:i + step].contiguous(), kt) / math.sqrt(case["dim"])
        s = s.masked_fill(~seen, -math.inf)
        e = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.matmul(e, vh) / e.sum(-1, keepdim=True)
        out[i:i + step] = o.transpose(0, 1).to(out.dtype)
    return out


def run(state):
    case = state["case"]
    if not state["own"]:
        return _plain_decode(state) if case["kind"] == "decode" else _plain_prefill(state)
    cache, kw = state["cache"], _window(case)
    if case["kind"] == "decode":
        return cache.attention(state["q"], seq_ids=state["ids"], **kw)
    if case["kind"] == "prefill":
        return cache.prefill(1, state["q"], **kw)
    cache.insert(1, *state["new"])
    o = cache.prefill(1, state["q"], **kw)
    cache.remove(1)
    return o


# -- the same in 64 bits -------------------------------------------------------


def _exact_rows(case, x):
    """What the cache stands for, rows [n, H, d] in float64."""
    x = x.double()
    if case["kv"] != "kv4":
        return x
    lo, hi = x.min(dim=2).values, x.max(dim=2).values
    # the scale is defined as an fp32 quotient kept in fp16
    step = (torch.div((hi - lo).float(), 15.0)).to(torch.float16).double().unsqueeze(2)
    lo = lo.unsqueeze(2)
    n = torch.where(step > 0, ((x - lo) / step).round(), torch.zeros((), dtype=torch.float64, device=x.device))
    return lo + step * torch.minimum(n, torch.full_like(n, 15.0))


def _exact_head(q, k, v, first, window, sinks):
    """One head: q [n, d] at positions first, first + 1, ...; k, v [L, d]."""
    at = first + torch.arange(q.shape[0], device=q.device)
    key = torch.arange(k.shape[0], device=q.device)
    gap = at[:, None] - key[None, :]
    hidden = gap < 0
    if window:
        hidden |= (gap >= window) & (key[None, :] >= sinks)
    s = (q.double() @ k.t()) * k.shape[1] ** -0.5
    return torch.softmax(s.masked_fill(hidden, -math.inf), dim=1) @ v


def exact(case, seed):
    w, s = case["window"], case["sinks"]
    if case["kind"] == "decode":
        segs, paths, q = _decode_inputs(case, seed)
        kv = [(_exact_rows(case, a[1]), _exact_rows(case, a[2])) if len(a[0]) else None for a in segs]
        out = torch.empty(q.shape, dtype=torch.float64, device=q.device)
        for r, path in enumerate(paths):
            k = torch.cat([kv[j][0] for j in path]).transpose(0, 1)
            v = torch.cat([kv[j][1] for j in path]).transpose(0, 1)
            L = k.shape[1]
            a = torch.matmul(k, q[r].double().unsqueeze(2)).squeeze(2) / math.sqrt(case["dim"])
            if w:
                a[:, s:max(s, L - w)] = -math.inf
            out[r] = torch.matmul(torch.softmax(a, dim=1).unsqueeze(1), v).squeeze(1)
        return out
    _, (_, k, v), q = _join_inputs(case, seed)
    n, H, d = q.shape
    out = torch.empty((n, H, d), dtype=torch.float64, device=q.device)
    for h in range(H):
        kh = _exact_rows(case, k[:, h:h + 1])[:, 0].contiguous()
        vh = _exact_rows(case, v[:, h:h + 1])[:, 0].contiguous()
        for i in range(0, n, 1024):
            out[i:i + 1024, h] = _exact_head(q[i:i + 1024, h], kh, vh, k.shape[0] - n + i, w, s)
    return out
