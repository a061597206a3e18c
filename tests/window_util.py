"""Shared by the tests of windowed attention and of the 4-bit cache."""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv4_values, window_attention, window_prefill
from paper_2402_15220_amd.cache import Cache
from parity_util import Pair, TORCH_DT, errors, to_dev, tol


class WPair(Pair):
    """The same cache on both sides, fp16, fp32 or (kv="kv4") 4-bit."""

    def __init__(self, c, H, d, kv, num_slots, layout="interleaved"):
        dtype = np.float32 if kv == "fp32" else np.float16
        super().__init__(c, H, d, dtype, 1, layout=layout)
        self.cache.close()
        self.kv = kv
        self.values = kv4_values if kv == "kv4" else None
        self.cache = Cache(c, H, d, num_slots, dtype=TORCH_DT[self.dtype], layout=layout,
                           kv_bits=4 if kv == "kv4" else None)

    def decode(self, q_by_sid, window=None, sinks=0, scale=0.0, seq_ids=None):
        """(o, reference), rows in the order asked for."""
        rows = self.cache.seq_order() if seq_ids is None else np.asarray(seq_ids)
        q = np.stack([q_by_sid[int(s)] for s in rows]).astype(self.dtype)
        out = torch.full(q.shape, float("nan"), dtype=TORCH_DT[self.dtype], device="cuda")
        o = self.cache.attention(to_dev(q), out=out, scale=scale, seq_ids=seq_ids, window=window, sinks=sinks)
        torch.cuda.synchronize()
        ref = window_attention(self.tree, rows, q, scale or 1 / np.sqrt(self.d), window, sinks, self.values)
        return o.cpu().numpy(), ref

    def prefill(self, sid, q, window=None, sinks=0, scale=0.0):
        out = torch.full(q.shape, float("nan"), dtype=TORCH_DT[self.dtype], device="cuda")
        o = self.cache.prefill(sid, to_dev(q), out=out, scale=scale, window=window, sinks=sinks)
        torch.cuda.synchronize()
        ref = window_prefill(self.tree, sid, q, scale or 1 / np.sqrt(self.d), window, sinks, self.values)
        return o.cpu().numpy(), ref


def assert_near(o, ref, dtype, what=""):
    """assert_close with the output's own rounding on top. The bar of
    assert_close is for averages over many N(0, 1) rows; a query that sees one
    to three tokens returns nearly a row itself, |o| up to 4.5 among 10^5 draws,
    and rounding that to fp16 alone is off by up to 2^-11 |o| = 2.2e-3, more
    than the whole bar of 2e-3. So 2^-11 |ref| is added to it."""
    _, rel, worst = errors(o, ref)
    amax, rmax = tol(dtype)
    over = np.abs(np.asarray(o, np.float64) - ref) - 2.0 ** -11 * np.abs(ref)
    print(f"[parity] {what} over own rounding={over.max():.3e} rel_l2={rel:.3e} worst_row={worst}", flush=True)
    assert over.max() <= amax and rel <= rmax, f"{what}: {over.max():.3e} rel_l2 {rel:.3e} (worst row {worst})"


def unpack_tile(tile, C, D):
    """Of one (slot, head) tile of a 4-bit pool: its codes [rows, D] read as a K
    tile and as a V tile, scale and low [rows]."""
    rows = -(-C // 16) * 16
    words = tile[: rows * D // 2].view(np.uint32)
    par = tile[rows * D // 2: rows * (D // 2 + 4)].view(np.float16).reshape(rows, 2)
    nib = np.array([(k >> 1) + 4 * (k & 1) for k in range(8)])
    k8 = (words[:, None] >> (4 * nib)[None, :]) & 15          # element k of every word
    # K: block, group g, token n, word w of the group: elements 8 (g D/32 + w) ..
    k_codes = k8.reshape(rows // 16, 4, 16, D // 32, 8).transpose(0, 2, 1, 3, 4).reshape(rows, D).astype(np.uint8)
    # V: block, group g, channel n, tile pair t; element 4 b + i is token 4 g + i, channel 32 t + 16 b + n
    v = k8.reshape(rows // 16, 4, 16, D // 32, 2, 4)
    v_codes = v.transpose(0, 1, 5, 3, 4, 2).reshape(rows, D).astype(np.uint8)
    return k_codes, v_codes, par[:, 0], par[:, 1]


def random_tree(p, rng, n_seqs=4, base_max=150, tail_max=200, gen=None):
    """n_seqs sequences that share prefixes of one base, some split mid-chunk;
    returns their token lists. Rows are N(0, 1), times `gen(n)` if given."""
    H, d = p.H, p.d
    base = rng.integers(0, 20, int(rng.integers(5, base_max))).astype(np.int32)
    seqs, kv = {}, {}
    for sid in range(n_seqs):
        cut = int(rng.integers(1, len(base) + 1))
        tail = rng.integers(20 + 40 * sid, 60 + 40 * sid, int(rng.integers(1, tail_max))).astype(np.int32)
        toks = np.concatenate([base[:cut], tail])
        k = rows_of(rng, kv, toks, H, d, p.dtype, 0)
        v = rows_of(rng, kv, toks, H, d, p.dtype, 1)
        p.insert(sid, toks, k, v)
        seqs[sid] = toks
    return seqs


def rows_of(rng, memo, toks, H, d, dtype, which):
    """Rows of a token list: equal prefixes have equal rows."""
    out = []
    key = (which,)
    for t in toks:
        key = (hash(key), int(t))
        if key not in memo:
            memo[key] = rng.standard_normal((H, d)).astype(dtype)
        out.append(memo[key])
    return np.stack(out)
