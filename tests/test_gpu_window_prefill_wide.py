"""Windowed prefill where the tiles are of 32-query wavefronts: whole tiles of
64 and 128 queries, chunks that fill a unit and chunks that do not, sinks and
window apart, rows that are not finite out of a query's sight."""
import numpy as np
import pytest
import torch

from oracle.window import _path
from parity_util import to_dev
from window_util import WPair, assert_near

pytestmark = pytest.mark.gpu


def head_ref(q, k, v, L, window, sinks):
    """One head in 64 bits: [n_q, d]; what a query does not see takes no part."""
    n_q, d = q.shape
    q, k, v = q.astype(np.float64), k.astype(np.float64), v.astype(np.float64)
    pos = np.arange(L - n_q, L)[:, None]
    j = np.arange(L)[None]
    see = (j <= pos) & ((j < sinks) | (j > pos - window))
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.where(see, q @ k.T / np.sqrt(d), -np.inf)
        m = s.max(1, keepdims=True)
        w = np.exp(s - m)
        n = w.sum(1, keepdims=True)
        fine = np.isfinite(v)
        o = (w @ np.where(fine, v, 0)) / n
        hit = (see.astype(np.float64) @ (~fine)) > 0
    return np.where(hit, np.nan, o)


def run(kv, H, d, c, L, n_q, window, sinks, bad, seed):
    print(f"[case] wide windowed prefill {kv} H={H} d={d} c={c} L={L} n_q={n_q} {window}+{sinks} {bad}", flush=True)
    rng = np.random.default_rng(seed)
    p = WPair(c, H, d, kv, (L + c - 1) // c + 1)
    k, v = (rng.standard_normal((L, H, d)).astype(np.float16) for _ in range(2))
    if bad is not None:
        for at in (0, 1, L // 2, L // 2 + 1, L - 100, L - 3):
            v[at, H - 1, at % d] = bad
    p.insert(0, np.arange(L, dtype=np.int32), k, v)
    kk, vv = _path(p.tree, 0, p.values)
    q = rng.standard_normal((n_q, H, d)).astype(np.float16)
    out = torch.full(q.shape, float("nan"), dtype=torch.float16, device="cuda")
    o = p.cache.prefill(0, to_dev(q), out=out, window=window, sinks=sinks).cpu().numpy()
    for h in (0, H - 1):
        ref = head_ref(q[:, h], kk[:, h], vv[:, h], L, window, sinks)
        ok = np.isfinite(ref)
        assert np.array_equal(np.isfinite(o[:, h]), ok), (h, np.argwhere(np.isfinite(o[:, h]) != ok)[:5])
        assert ok.any() or (kv == "kv4" and sinks)  # there a row among the sinks is NaN throughout
        if not ok.any():
            continue
        assert_near(o[:, h][ok][None], ref[ok][None], np.float16, f"head {h}")
    p.cache.close()


# (heads, d, chunk, length, queries): 256 tiles of 128, or of 64 queries and more
# than 256 of those; a chunk of 16 and 32 shares its unit, one of 40 does not
# fill it, one of 200 has four
SHAPES = [(16, 128, 64, 2300, 2000), (16, 128, 16, 2200, 2048), (16, 128, 32, 2100, 2100), (16, 128, 40, 2050, 2040),
          (16, 128, 200, 2300, 2000), (10, 128, 64, 1900, 1900), (10, 128, 16, 1800, 1777), (10, 128, 32, 1900, 1801),
          (34, 64, 64, 3500, 2049), (20, 64, 32, 2100, 2100), (16, 64, 64, 2200, 2100), (16, 64, 16, 2100, 2099),
          (16, 64, 200, 2100, 2050)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("window,sinks", [(77, 3), (700, 130), (5000, 0)])
def test_windows(shape, window, sinks):
    run("fp16", *shape, window, sinks, None, 41)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("bad", [np.inf, np.nan])
def test_not_finite(shape, bad):
    run("fp16", *shape, 333, 5, bad, 42)


@pytest.mark.parametrize("shape", [SHAPES[i] for i in (0, 1, 3, 5, 8, 10)])
@pytest.mark.parametrize("bad,sinks", [(None, 5), (np.nan, 5), (np.nan, 0)])
def test_4_bits(shape, bad, sinks):
    run("kv4", *shape, 333, sinks, bad, 43)
