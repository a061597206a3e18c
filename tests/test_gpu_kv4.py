"""GPU tests of the cache held in 4 bits: the stored codes against the
definition, decode attention against the float64 oracle over the values that
the codes stand for, growth, splits, removal, refusals."""
import numpy as np
import pytest
import torch

from oracle import kv4_quantise
from paper_2402_15220_amd.cache import Cache
from paper_2402_15220_amd.binding import ChunkAttnError
from parity_util import assert_close, to_dev
from window_util import WPair, random_tree, rows_of, unpack_tile

pytestmark = pytest.mark.gpu


def check_tiles(p):
    """Codes and parameters of every stored row equal the definition's."""
    torch.cuda.synchronize()
    kp, vp = p.cache.k_pool.cpu().numpy(), p.cache.v_pool.cpu().numpy()
    for n in p.tree.nodes():
        L = len(n)
        for h in range(p.H):
            for pool, rows, which in ((kp, n.k, 0), (vp, n.v, 1)):
                got = unpack_tile(np.ascontiguousarray(pool[n.slot, h]), p.c, p.d)
                code, scale, low = kv4_quantise(rows[:, h])
                assert np.array_equal(got[which][:L], code), (n.slot, h, which)
                assert np.array_equal(got[2][:L], scale[:, 0], equal_nan=True)
                assert np.array_equal(got[3][:L], low[:, 0], equal_nan=True)


@pytest.mark.parametrize("c,d,layout", [(1, 64, "interleaved"), (7, 128, "split"), (16, 64, "interleaved"),
                                        (64, 128, "interleaved"), (33, 128, "split"), (100, 64, "interleaved")])
def test_stored_codes(c, d, layout):
    """Inserts, splits inside a chunk, single-token appends into partly filled
    16-token blocks, extends across chunks, slots used again."""
    print(f"[case] kv4 codes c={c} d={d}", flush=True)
    rng = np.random.default_rng(c)
    H = 3
    p = WPair(c, H, d, "kv4", 1200, layout=layout)
    seqs = random_tree(p, rng)
    check_tiles(p)
    for step in range(5):
        ids = list(seqs)
        k, v = (rng.standard_normal((len(ids), H, d)).astype(np.float16) for _ in range(2))
        p.append(ids, rng.integers(0, 9, len(ids)).astype(np.int32), k, v)
    n = 2 * c + 3
    p.extend(1, rng.integers(0, 99, n).astype(np.int32),
             *(rng.standard_normal((n, H, d)).astype(np.float16) for _ in range(2)))
    check_tiles(p)
    p.remove(0)
    memo = {}
    toks = np.arange(500, 500 + 40, dtype=np.int32)
    p.insert(9, toks, rows_of(rng, memo, toks, H, d, np.float16, 0), rows_of(rng, memo, toks, H, d, np.float16, 1))
    check_tiles(p)


def test_codes_of_special_rows():
    """Constant rows, rows of two neighbouring values, subnormal spreads, the
    largest spread, ties between codes, non-finite elements."""
    print("[case] kv4 special rows", flush=True)
    d, H, c = 128, 1, 16
    rng = np.random.default_rng(0)
    x = rng.standard_normal((24, H, d)).astype(np.float16)
    x[0] = 0
    x[1] = -3.5
    x[2, 0] = np.where(np.arange(d) % 2, np.float16(1), np.nextafter(np.float16(1), np.float16(2)))
    x[3, 0] = (np.arange(d) % 5) * np.float16(2.0 ** -24)
    x[4, 0, 0], x[4, 0, 1] = 65504, -65504
    x[5, 0] = (np.arange(d) % 31) / np.float16(2)   # scale 1: every odd half is a tie
    x[6, 0] = -(np.arange(d) % 31) / np.float16(2)
    x[7, 0, 5] = np.inf
    x[8, 0, 127] = -np.inf
    x[9, 0, 64] = np.nan
    x[10, 0] = rng.standard_normal(d) * 2.0 ** -14
    x[11] = x[11] * 60
    p = WPair(c, H, d, "kv4", 8)
    p.insert(0, np.arange(24, dtype=np.int32), x, x[::-1].copy())
    check_tiles(p)


@pytest.mark.parametrize("case", range(10))
def test_decode_random_trees(case):
    c = [64, 16, 1, 7, 100, 64, 32, 17, 128, 48][case]
    d = [128, 64][case % 2]
    H = [4, 1, 3, 2, 5][case % 5]
    rng = np.random.default_rng(700 + case)
    print(f"[case] kv4 decode c={c} d={d} H={H}", flush=True)
    p = WPair(c, H, d, "kv4", 4096, layout=["interleaved", "split"][case % 3 == 1])
    seqs = random_tree(p, rng, n_seqs=[4, 1, 6, 23][case % 4], base_max=400, tail_max=300)
    q = {s: rng.standard_normal((H, d)).astype(np.float16) for s in seqs}
    o, ref = p.decode(q)
    assert_close(o, ref, np.float16, f"kv4 c={c} d={d}")
    order = list(rng.permutation(list(seqs)))
    o, ref = p.decode(q, seq_ids=order, scale=0.3)
    assert_close(o, ref, np.float16, f"kv4 ordered c={c} d={d}")
    # decode steps: growth into new chunks, then a leave and a join
    for step in range(3):
        ids = list(seqs)
        p.append(ids, np.full(len(ids), 7 + step, np.int32),
                 *(rng.standard_normal((len(ids), H, d)).astype(np.float16) for _ in range(2)))
        o, ref = p.decode(q)
        assert_close(o, ref, np.float16, f"kv4 step {step} c={c} d={d}")
    if len(seqs) > 1:
        p.remove(0)
        o, ref = p.decode(q)
        assert_close(o, ref, np.float16, f"kv4 after a leave c={c} d={d}")


def test_identical_sequences_and_one_token():
    """Shared chunks only (more rows than one tile), then a single token."""
    print("[case] kv4 identical sequences", flush=True)
    rng = np.random.default_rng(3)
    H, d = 2, 128
    p = WPair(64, H, d, "kv4", 64)
    n = 700
    k, v = (rng.standard_normal((n, H, d)).astype(np.float16) for _ in range(2))
    for sid in range(37):
        p.insert(sid, np.arange(n, dtype=np.int32), k, v)
    q = {s: rng.standard_normal((H, d)).astype(np.float16) for s in range(37)}
    o, ref = p.decode(q)
    assert_close(o, ref, np.float16, "kv4 37 identical rows")
    p1 = WPair(64, H, d, "kv4", 4)
    p1.insert(5, [3], k[:1], v[:1])
    o, ref = p1.decode({5: q[0]})
    assert_close(o, ref, np.float16, "kv4 one token")


@pytest.mark.parametrize("spread", [2.0 ** -12, 1.0, 100.0, 400.0])
def test_decode_scales_of_rows(spread):
    """Rows whose scales differ by orders of magnitude: V weights are formed
    relative to a running reference of the scales, small and large first. At
    the largest spread some elements overflow to infinity: the result is NaN."""
    print(f"[case] kv4 scales {spread}", flush=True)
    rng = np.random.default_rng(11)
    H, d, n = 2, 64, 333
    p = WPair(64, H, d, "kv4", 32)
    k = rng.standard_normal((n, H, d)).astype(np.float16)
    mag = np.exp2(rng.uniform(-6, 6, (n, H, 1))) * spread
    with np.errstate(over="ignore"):
        v = (rng.standard_normal((n, H, d)) * mag).astype(np.float16)
    p.insert(0, np.arange(n, dtype=np.int32), k, v)
    o, ref = p.decode({0: rng.standard_normal((H, d)).astype(np.float16)})
    # Relative to the largest value: each of the n weights is rounded to fp16
    # (2^-11) and scales a code of at most 8 steps; |o| errors add up to at
    # most sum p 2^-11 8 s <= 2^-11 8 max(s), plus o's own rounding, 2^-11 |o|;
    # below the normal range fp16 steps are 2^-24 and a half step is added.
    if spread == 400.0:
        assert np.isinf(v).any() and np.isnan(ref).all() and np.isnan(o).all()
        return
    s = kv4_quantise(v)[1].astype(np.float64).max()
    assert np.abs(o - ref).max() <= 2.0 ** -11 * (8 * s + np.abs(ref).max()) + 2.0 ** -25


def test_large_queries_and_extreme_values():
    """q far outside [-1, 1] and subnormal q; masked-out garbage in the pool
    (NaN patterns behind the last row) does not reach o."""
    print("[case] kv4 extremes", flush=True)
    rng = np.random.default_rng(12)
    H, d, n = 2, 128, 77
    p = WPair(64, H, d, "kv4", 16)
    p.cache.kv_pool.fill_(0xFF)  # codes 15, scale and low NaN
    k, v = (rng.standard_normal((n, H, d)).astype(np.float16) for _ in range(2))
    p.insert(0, np.arange(n, dtype=np.int32), k, v)
    for mul in (1e3, 1.0, 1e-7):
        q = (rng.standard_normal((H, d)) * mul).astype(np.float16)
        o, ref = p.decode({0: q}, scale=1.0 / (max(mul, 1.0) * 11))
        assert_close(o, ref, np.float16, f"kv4 q x {mul}")


def test_noalloc_and_graph_replay():
    """ca_attention_noalloc, and a call captured into a graph whose replays
    follow appends that only fill chunks."""
    print("[case] kv4 noalloc, graph", flush=True)
    rng = np.random.default_rng(13)
    H, d = 4, 128
    p = WPair(64, H, d, "kv4", 256)
    seqs = random_tree(p, rng, n_seqs=5, base_max=300, tail_max=50)
    # sequences of their own for the appends, far from the end of a chunk
    q = {s: rng.standard_normal((H, d)).astype(np.float16) for s in seqs}
    p.cache.prepare()
    rows = p.cache.seq_order()
    qd = to_dev(np.stack([q[int(s)] for s in rows]))
    o0, ref = p.decode(q)
    out = torch.full_like(qd, float("nan"))
    p.cache.attention_noalloc(qd, out)
    torch.cuda.synchronize()
    assert_close(out.cpu().numpy(), ref, np.float16, "kv4 noalloc")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        p.cache.attention(qd, out=out)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            p.cache.attention(qd, out=out)
        for step in range(3):
            out.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            ref = p.decode(q)[1]
            assert_close(out.cpu().numpy(), ref, np.float16, f"kv4 replay {step}")
            fits = [s for s in seqs if len(p.tree.path(s)[-1]) < 60 and _private(p, s)]
            before = p.cache.stats()["slots_used"]
            if fits:
                p.append(fits, np.full(len(fits), 3, np.int32),
                         *(rng.standard_normal((len(fits), H, d)).astype(np.float16) for _ in range(2)))
            assert p.cache.stats()["slots_used"] == before


def _private(p, sid):
    leaf = p.tree.path(sid)[-1]
    return sum(leaf in p.tree.path(s) for s in p.tree.seq_ids()) == 1


def test_refusals():
    with pytest.raises(ValueError):
        Cache(64, 2, 64, 8, dtype=torch.float32, kv_bits=4)
    with pytest.raises(ValueError):
        Cache(64, 2, 64, 8, kv_bits=8)
    c = Cache(64, 2, 64, 8, kv_bits=4)
    kv = torch.zeros(4, 2, 64, dtype=torch.float32, device="cuda")
    with pytest.raises(ValueError):
        c.insert(0, [1, 2, 3, 4], kv, kv)
    kv = kv.half()
    c.insert(0, [1, 2, 3, 4], kv, kv)
    out = torch.empty(1, 2, 64, dtype=torch.float16, device="cuda")
    with pytest.raises(ChunkAttnError):  # context not current
        c.attention_noalloc(kv[:1].contiguous(), out)
    c.close()
