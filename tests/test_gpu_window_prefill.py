"""GPU tests of prefill with a sliding window and sinks, over fp16 and 4-bit
pools (and of a 4-bit pool's prefill without a window), against the float64
oracle; the joins and decode steps of a served batch over a 4-bit, windowed
cache as one run."""
import numpy as np
import pytest
import torch

from paper_2402_15220_amd.binding import ChunkAttnError
from paper_2402_15220_amd.cache import Cache
from parity_util import to_dev
from window_util import WPair, assert_near, random_tree, rows_of

pytestmark = pytest.mark.gpu

KINDS = ["fp16", "kv4"]


@pytest.mark.parametrize("kv", KINDS)
@pytest.mark.parametrize("case", range(10))
def test_random_trees(kv, case):
    rng = np.random.default_rng(1500 + case)
    c = [1, 3, 16, 64, 5, 64, 32, 128, 100, 65][case]
    d = [64, 128][(case + KINDS.index(kv)) % 2]
    H = 1 + case % 3
    print(f"[case] window prefill {kv} c={c} d={d} H={H}", flush=True)
    p = WPair(c, H, d, kv, 4096, layout=["interleaved", "split"][case % 4 == 3])
    seqs = random_tree(p, rng, n_seqs=3)
    for sid, toks in seqs.items():
        L = len(toks)
        for n_q in sorted({1, min(L, 5), min(L, 63), min(L, 65), min(L, 130), L}):
            q = rng.standard_normal((n_q, H, d)).astype(np.float16)
            for window, sinks in ((1, 0), (1, 2), (40, 3), (64, 0), (129, 20), (L, 1), (10 ** 12, 0)):
                o, ref = p.prefill(sid, q, window, sinks, scale=0.0 if n_q % 2 else 0.2)
                assert_near(o, ref, np.float16, f"{kv} c={c} d={d} L={L} n_q={n_q} window={window} sinks={sinks}")
            if kv == "kv4":
                o, ref = p.prefill(sid, q)
                assert_near(o, ref, np.float16, f"{kv} c={c} d={d} L={L} n_q={n_q}")


@pytest.mark.parametrize("kv", KINDS)
@pytest.mark.parametrize("H,c,L,n_q,window,sinks", [(40, 64, 900, 777, 300, 4), (2, 64, 5000, 100, 4500, 100),
                                                    (1, 16, 5000, 33, 4700, 0), (3, 64, 20000, 64, 18000, 3)])
def test_large(kv, H, c, L, n_q, window, sinks):
    """128-query tiles, parts of a tile's keys, paths of more than 255 chunks."""
    print(f"[case] window prefill large {kv} H={H} c={c} L={L} n_q={n_q}", flush=True)
    rng = np.random.default_rng(L)
    d = 128
    p = WPair(c, H, d, kv, -(-L // c) + 4)
    p.insert(0, np.arange(L, dtype=np.int32), *(rng.standard_normal((L, H, d)).astype(np.float16) for _ in range(2)))
    q = rng.standard_normal((n_q, H, d)).astype(np.float16)
    keep = rng.choice(n_q, min(n_q, 12), replace=False)
    for w, s in ((window, sinks), (10 ** 9, 0)):
        out = torch.full(q.shape, float("nan"), dtype=torch.float16, device="cuda")
        p.cache.prefill(0, to_dev(q), out=out, window=w, sinks=s)
        torch.cuda.synchronize()
        o = out.cpu().numpy()
        assert np.isfinite(o).all()
        from oracle.window import _path, visible
        from oracle.attention import _softmax_attend
        k, v = _path(p.tree, 0, p.values)
        for i in keep:
            j = visible(L - n_q + i, w, s)
            ref = _softmax_attend(q[i].astype(np.float64), k[j], v[j], 1 / np.sqrt(d))
            assert_near(o[i:i + 1], ref[None], np.float16, f"{kv} L={L} query {i} window={w}")


@pytest.mark.parametrize("kv", KINDS)
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_non_finite_out_of_sight(kv, bad):
    """Non-finite K and V rows: queries before them, or past them by more than
    the window, are right; queries that see them are not finite there."""
    print(f"[case] window prefill non-finite {kv} {bad}", flush=True)
    rng = np.random.default_rng(31)
    H, d, c, L = 2, 64, 64, 300
    p = WPair(c, H, d, kv, 16)
    k, v = (rng.standard_normal((L, H, d)).astype(np.float16) for _ in range(2))
    v[100, :, 5] = bad
    v[101, 0, 40] = bad
    k[180, 1, 3] = np.nan if np.isnan(bad) else bad
    p.insert(0, np.arange(L, dtype=np.int32), k, v)
    for n_q, window, sinks in ((300, 37, 2), (250, 1, 0), (300, 64, 101), (130, 60, 0)):
        q = rng.standard_normal((n_q, H, d)).astype(np.float16)
        with np.errstate(invalid="ignore"):
            o, ref = p.prefill(0, q, window, sinks)
        ok = np.isfinite(ref)
        assert np.array_equal(np.isfinite(o), ok), (n_q, window, sinks)
        assert_near(o[ok][None], ref[ok][None], np.float16, f"{kv} n_q={n_q} window={window}")


@pytest.mark.parametrize("kv", KINDS)
def test_garbage_behind_the_rows(kv):
    print(f"[case] window prefill garbage {kv}", flush=True)
    rng = np.random.default_rng(32)
    p = WPair(37, 2, 128, kv, 64)
    p.cache.kv_pool.view(torch.uint8).fill_(0xFF)
    seqs = random_tree(p, rng, n_seqs=3, base_max=80, tail_max=100)
    for sid, toks in seqs.items():
        q = rng.standard_normal((len(toks), 2, 128)).astype(np.float16)
        for window, sinks in ((50, 3), (1000, 0)):
            o, ref = p.prefill(sid, q, window, sinks)
            assert_near(o, ref, np.float16, f"garbage {kv}")


@pytest.mark.parametrize("kv", KINDS)
def test_captured_prefill(kv):
    """Replays of a captured call equal the eager one; a path of more than 255
    chunks is refused under capture, and a window that sees fewer is not."""
    print(f"[case] window prefill graph {kv}", flush=True)
    rng = np.random.default_rng(33)
    H, d, c, L = 2, 64, 16, 6000
    p = WPair(c, H, d, kv, 400)
    p.insert(0, np.arange(L, dtype=np.int32), *(rng.standard_normal((L, H, d)).astype(np.float16) for _ in range(2)))
    q = to_dev(rng.standard_normal((70, H, d)).astype(np.float16))
    out = torch.empty_like(q)
    want = p.cache.prefill(0, q, window=2000, sinks=5).clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        p.cache.prefill(0, q, out=out, window=2000, sinks=5)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            p.cache.prefill(0, q, out=out, window=2000, sinks=5)
            with pytest.raises(ChunkAttnError):
                p.cache.prefill(0, q, out=torch.empty_like(q), window=5000)
        for _ in range(3):
            out.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            assert torch.equal(p.cache.prefill(0, q, window=2000, sinks=5), want)


@pytest.mark.parametrize("kv", KINDS)
def test_served_batch(kv):
    """Joins behind a shared prompt, windowed decode steps, leaves and a late
    join: writes, prefill and decode together."""
    print(f"[case] served batch {kv}", flush=True)
    rng = np.random.default_rng(34)
    H, d, c, window, sinks = 4, 128, 64, 150, 4
    p = WPair(c, H, d, kv, 256)
    memo = {}
    prompt = rng.integers(0, 1000, 200).astype(np.int32)

    def join(sid, n):
        toks = np.concatenate([prompt, 2000 + 100 * sid + np.arange(n, dtype=np.int32)])
        m = p.insert(sid, toks, rows_of(rng, memo, toks, H, d, np.float16, 0),
                     rows_of(rng, memo, toks, H, d, np.float16, 1))
        q = rng.standard_normal((len(toks) - m, H, d)).astype(np.float16)
        for w, s in ((window, sinks), (10 ** 9, 0)):
            o, ref = p.prefill(sid, q, w, s)
            assert_near(o, ref, np.float16, f"{kv} join {sid} window={w}")

    for sid in range(4):
        join(sid, 5 + 17 * sid)
    live = [0, 1, 2, 3]
    for step in range(30):
        p.append(live, rng.integers(0, 99, len(live)).astype(np.int32),
                 *(rng.standard_normal((len(live), H, d)).astype(np.float16) for _ in range(2)))
        q = {s: rng.standard_normal((H, d)).astype(np.float16) for s in live}
        o, ref = p.decode(q, window, sinks, seq_ids=live)
        assert_near(o, ref, np.float16, f"{kv} step {step}")
        o, ref = p.decode(q)  # a layer that sees everything, by turns
        assert_near(o, ref, np.float16, f"{kv} step {step} full")
        if step == 10:
            p.remove(1)
            live.remove(1)
            join(7, 33)
            live.append(7)


def test_refusals():
    c = Cache(64, 2, 64, 8)
    kv = torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda")
    c.insert(0, [1, 2, 3, 4], kv, kv)
    for window, sinks in ((0, 0), (-1, 0), (4, -1)):
        with pytest.raises(ChunkAttnError):
            c.prefill(0, kv, window=window, sinks=sinks)
    with pytest.raises(ValueError):
        c.prefill(0, kv, sinks=3)
    with pytest.raises(ChunkAttnError):
        c.prefill(1, kv, window=3)
    with pytest.raises(ChunkAttnError):
        c.prefill(0, torch.zeros(5, 2, 64, dtype=torch.float16, device="cuda"), window=3)
    assert c.prefill(0, kv[:0], window=3).shape == (0, 2, 64)
    c.close()
    c = Cache(64, 2, 64, 8, dtype=torch.float32)
    kv = kv.float()
    c.insert(0, [1, 2, 3, 4], kv, kv)
    with pytest.raises(ChunkAttnError):
        c.prefill(0, kv, window=3)
    c.close()
