"""GPU tests of the cache held in 4 bits: the stored codes against the
definition, decode attention against the float64 oracle over the values that
the codes stand for, growth, splits, removal, refusals."""
import numpy as np
import pytest
import torch

from oracle import kv4_quantise, kv4_values
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


def _prefill_ref(q, k, v, scale):
    """Causal, every head, in 64 bits: [n_q, H, d]."""
    n_q, L = q.shape[0], k.shape[0]
    s = scale * np.einsum("qhd,lhd->hql", q.astype(np.float64), k)
    s = np.where(np.arange(L)[None, None] <= (L - n_q + np.arange(n_q))[None, :, None], s, -np.inf)
    w = np.exp(s - s.max(-1, keepdims=True))
    return np.einsum("hql,lhd->qhd", w / w.sum(-1, keepdims=True), v)


def _prefill_bar(q, k, v, scale, step):
    """What rounding can do, [n_q, H, 1]. A weight p is rounded to fp16 (2^-11)
    and scales up to 8 steps of its row (at most `step` each), and o is rounded (2^-11), half a step
    of the subnormal range where that is larger. A score is the sum of
    q s^(code - 8) and b sum(q), each at most max|k| sum|q| in size, over d + 8
    products that fp32 accumulates, off by at most 2^-23 of the running sum at
    each: e = scale 2 max|k| sum|q| (d + 8) 2^-23, which moves weights by a
    factor e^(+-2e) and so o by at most 2 e max|v - o| <= 4 e max|v|."""
    d = q.shape[2]
    e = scale * 2 * np.abs(k).max() * np.abs(q.astype(np.float64)).sum(-1, keepdims=True) * (d + 8) * 2.0 ** -23
    return 2.0 ** -11 * (8 * step + np.abs(v).max()) + 4 * e * np.abs(v).max() + 2.0 ** -25


def _extreme_rows(rng, n, H, d, kind):
    x = rng.standard_normal((n, H, d))
    if kind == "wide":  # some rows over nearly all of fp16's range
        x[::7] = np.clip(x[::7] * 3e4, -65504, 65504)
        x[3, :, :2] = (-65504, 65504)
    elif kind == "end":  # rows at an end of it, and constant ones
        x[::5] = 65472 + 32 * (rng.random((len(x[::5]), H, d)) > 0.5)
        x[2::5] = -65504
    elif kind == "small":  # subnormal values and scales
        x *= 1e-6
        x[1::3] *= 0
    elif kind == "mixed":  # scales over orders of magnitude
        x *= np.exp2(rng.uniform(-20, 12, (n, H, 1)))
    return x.astype(np.float16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k_kind,v_kind,q_mul,scale", [
    ("wide", "normal", 1e-4, 0.1), ("end", "normal", 1e-4, 0.1), ("small", "normal", 1e3, 0.1),
    ("mixed", "normal", 1e-2, 0.1), ("normal", "wide", 1.0, 0.1), ("normal", "end", 1.0, 0.1),
    ("normal", "small", 1.0, 0.1), ("normal", "mixed", 1.0, 0.1), ("normal", "wide", 1.0, 1e-8),
    ("normal", "normal", 1e-3, 1e2), ("end", "end", 1e-5, 1.0), ("normal", "normal", 1.0, 50.0)])
def test_prefill_extremes(d, k_kind, v_kind, q_mul, scale):
    print(f"[case] kv4 prefill extremes d={d} {k_kind} {v_kind} {q_mul} {scale}", flush=True)
    rng = np.random.default_rng(21)
    H, n, n_q = 2, 300, 150
    p = WPair(64, H, d, "kv4", 16)
    k, v = _extreme_rows(rng, n, H, d, k_kind), _extreme_rows(rng, n, H, d, v_kind)
    p.insert(0, np.arange(n, dtype=np.int32), k, v)
    q = (rng.standard_normal((n_q, H, d)) * q_mul).astype(np.float16)
    o = p.cache.prefill(0, to_dev(q), scale=scale).cpu().numpy()
    kk, vv = kv4_values(k).astype(np.float64), kv4_values(v).astype(np.float64)
    err = np.abs(o - _prefill_ref(q, kk, vv, scale))
    bar = _prefill_bar(q, kk, vv, scale, kv4_quantise(v)[1].astype(np.float64).max())
    assert (err <= bar).all(), (err.max(), bar.min())


def test_prefill_large_sums_of_q():
    """Queries whose elements add up to more than fp16 holds, in one tile with
    queries of ordinary and of tiny elements."""
    print("[case] kv4 prefill sums of q", flush=True)
    rng = np.random.default_rng(22)
    H, d, n = 2, 128, 200
    for k_mul, scale in ((1.0, 1e-4), (3e3, 1.0)):
        p = WPair(64, H, d, "kv4", 16)
        k = (rng.standard_normal((n, H, d)) * k_mul).astype(np.float16)
        v = rng.standard_normal((n, H, d)).astype(np.float16)
        p.insert(0, np.arange(n, dtype=np.int32), k, v)
        q = rng.standard_normal((n, H, d)).astype(np.float16)
        q[::3] = 1000 + 10 * q[::3]
        q[1::3] *= np.float16(1e-4)
        o = p.cache.prefill(0, to_dev(q), scale=scale).cpu().numpy()
        kk, vv = kv4_values(k).astype(np.float64), kv4_values(v).astype(np.float64)
        err = np.abs(o - _prefill_ref(q, kk, vv, scale))
        bar = _prefill_bar(q, kk, vv, scale, kv4_quantise(v)[1].astype(np.float64).max())
        assert np.isfinite(o).all() and (err <= bar).all(), (err.max(), bar.min())
        # the tiny ones' bar is their own, not the large ones': sum|q| = 0.0104,
        # max|k| = 1.4e4: e = 2 * 1.4e4 * 0.0104 * 136 / 2^23 = 4.7e-3, times
        # 4 max|v| = 17.6 0.083, and the weights' 2^-11 (8 * 0.6 + 4.4) = 0.005
        assert bar[1::3].max() < 0.1 and (err[1::3] < 0.1).all()


def test_prefill_scale_refused():
    c = Cache(64, 2, 64, 8, kv_bits=4)
    kv = torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda")
    c.insert(0, [1, 2, 3, 4], kv, kv)
    for scale in (1e-12, 1e9, float("nan"), float("inf"), -1.0):
        with pytest.raises(ChunkAttnError):
            c.prefill(0, kv, scale=scale)
    c.close()


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
