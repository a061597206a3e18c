"""GPU tests of decode attention with a sliding window and sinks against the
float64 oracle: random trees over every storage, window and sink counts around
tile, chunk and sequence lengths, growth, non-finite values out of sight."""
import numpy as np
import pytest
import torch

from paper_2402_15220_amd import binding
from paper_2402_15220_amd.binding import ChunkAttnError
from paper_2402_15220_amd.cache import Cache
from parity_util import assert_close, to_dev
from window_util import WPair, random_tree

pytestmark = pytest.mark.gpu

KINDS = ["fp16", "fp32", "kv4"]


@pytest.mark.parametrize("kv", KINDS)
@pytest.mark.parametrize("case", range(8))
def test_random_trees(kv, case):
    c = [64, 16, 5, 100, 64, 32, 1, 128][case]
    d = [128, 64][(case + KINDS.index(kv)) % 2]
    H = [3, 1, 2, 4][case % 4]
    rng = np.random.default_rng(900 + case)
    print(f"[case] window decode {kv} c={c} d={d} H={H}", flush=True)
    p = WPair(c, H, d, kv, 4096, layout=["interleaved", "split"][case % 2])
    seqs = random_tree(p, rng, n_seqs=[5, 20, 2, 9][case % 4], base_max=300, tail_max=250)
    q = {s: rng.standard_normal((H, d)).astype(p.dtype) for s in seqs}
    longest = max(len(t) for t in seqs.values())
    for window, sinks in ((1, 0), (1, 1), (2, 3), (16, 0), (17, 4), (c, 1), (100, 16), (longest - 1, 2),
                          (longest, 0), (10 ** 12, 5), (3, 10 ** 12)):
        o, ref = p.decode(q, window, sinks)
        assert_close(o, ref, p.dtype, f"{kv} c={c} d={d} window={window} sinks={sinks}")
    order = list(rng.permutation(list(seqs)))
    for step in range(4):
        o, ref = p.decode(q, 40, 2, scale=0.21, seq_ids=order)
        assert_close(o, ref, p.dtype, f"{kv} ordered step {step} c={c} d={d}")
        p.append(order, np.full(len(order), 5 + step, np.int32),
                 *(rng.standard_normal((len(order), H, d)).astype(p.dtype) for _ in range(2)))
    # windows by turns, full attention between them
    for window in (40, None, 30, 40):
        o, ref = p.decode(q, window, 2 if window else 0)
        assert_close(o, ref, p.dtype, f"{kv} in turn window={window}")


@pytest.mark.parametrize("kv", KINDS)
def test_window_moves_over_many_steps(kv):
    """Single appends past several chunk ends: the context is patched, and the
    window's start passes chunk and tile borders."""
    print(f"[case] window growth {kv}", flush=True)
    rng = np.random.default_rng(21)
    H, d, c = 2, 64, 16
    p = WPair(c, H, d, kv, 256)
    seqs = random_tree(p, rng, n_seqs=3, base_max=60, tail_max=40)
    q = {s: rng.standard_normal((H, d)).astype(p.dtype) for s in seqs}
    for step in range(70):
        p.append(list(seqs), np.full(3, step, np.int32),
                 *(rng.standard_normal((3, H, d)).astype(p.dtype) for _ in range(2)))
        o, ref = p.decode(q, 33, 2)
        assert_close(o, ref, p.dtype, f"{kv} step {step}")


@pytest.mark.parametrize("kv", KINDS)
def test_long_rows(kv):
    """Many items a row: a long private row beside short ones."""
    print(f"[case] window long {kv}", flush=True)
    rng = np.random.default_rng(22)
    H, d, c = 2, 128, 64
    p = WPair(c, H, d, kv, 400)
    lens = [9001, 1, 640, 63]
    for s, n in enumerate(lens):
        p.insert(s, np.arange(10000 * s, 10000 * s + n, dtype=np.int32),
                 *(rng.standard_normal((n, H, d)).astype(p.dtype) for _ in range(2)))
    q = {s: rng.standard_normal((H, d)).astype(p.dtype) for s in range(4)}
    for window, sinks in ((8000, 4), (4096, 0), (100, 700), (20000, 0)):
        o, ref = p.decode(q, window, sinks)
        assert_close(o, ref, p.dtype, f"{kv} long window={window} sinks={sinks}")


@pytest.mark.parametrize("kv", KINDS)
@pytest.mark.parametrize("bad", [np.inf, np.nan])
def test_non_finite_out_of_sight(kv, bad):
    """A shared chunk whose start has left some rows' windows but not others',
    with non-finite K and V rows there: rows that do not see them are right,
    rows that do are not finite."""
    print(f"[case] window non-finite {kv} {bad}", flush=True)
    rng = np.random.default_rng(23)
    H, d, c = 2, 64, 64
    p = WPair(c, H, d, kv, 64)
    base = np.arange(64, dtype=np.int32)
    kb, vb = (rng.standard_normal((64, H, d)).astype(p.dtype) for _ in range(2))
    kb[20, :, 3] = bad
    vb[21, :, 5] = bad
    vb[60, :, 7] = bad       # hidden from the longest row only
    lens = {0: 1, 1: 30, 2: 90, 3: 33, 4: 34}
    for s, n in lens.items():
        kt, vt = (rng.standard_normal((n, H, d)).astype(p.dtype) for _ in range(2))
        p.insert(s, np.concatenate([base, 100 + 200 * s + np.arange(n, dtype=np.int32)]),
                 np.concatenate([kb, kt]), np.concatenate([vb, vt]))
    q = {s: rng.standard_normal((H, d)).astype(p.dtype) for s in lens}
    with np.errstate(invalid="ignore", over="ignore"):
        for window, sinks in ((75, 0), (90, 2), (30, 0), (36, 4), (92, 0)):
            rows = p.cache.seq_order()
            o, ref = p.decode(q, window, sinks)
            ok = np.isfinite(ref)
            assert np.array_equal(np.isfinite(o), ok), (window, sinks)
            if ok.any():
                assert_close(o[ok][None], ref[ok][None], p.dtype, f"{kv} window={window} sinks={sinks} rows={rows}")


def test_garbage_behind_the_rows():
    """Pools filled with NaN before use: unused rows of partly filled chunks
    and of tiles past a chunk's end add nothing."""
    print("[case] window garbage", flush=True)
    rng = np.random.default_rng(24)
    for kv in KINDS:
        p = WPair(37, 2, 128, kv, 64)
        p.cache.kv_pool.view(torch.uint8).fill_(0xFF)
        seqs = random_tree(p, rng, n_seqs=5, base_max=80, tail_max=60)
        q = {s: rng.standard_normal((2, 128)).astype(p.dtype) for s in seqs}
        for window, sinks in ((50, 3), (1000, 0)):
            o, ref = p.decode(q, window, sinks)
            assert_close(o, ref, p.dtype, f"garbage {kv}")


def test_graph_replay_follows_appends():
    """A captured windowed call: replays after appends that fill chunks see the
    window moved; a call that would have to upload is refused under capture."""
    print("[case] window graph", flush=True)
    rng = np.random.default_rng(25)
    H, d = 2, 64
    for kv in KINDS:
        p = WPair(64, H, d, kv, 64)
        for s, n in enumerate((70, 5, 130)):
            p.insert(s, np.arange(1000 * s, 1000 * s + n, dtype=np.int32),
                     *(rng.standard_normal((n, H, d)).astype(p.dtype) for _ in range(2)))
        q = {s: rng.standard_normal((H, d)).astype(p.dtype) for s in range(3)}
        rows = p.cache.seq_order()
        qd = to_dev(np.stack([q[int(s)] for s in rows]))
        out = torch.empty_like(qd)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            p.cache.attention(qd, out=out, window=20, sinks=1)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                p.cache.attention(qd, out=out, window=20, sinks=1)
                with pytest.raises(ChunkAttnError):
                    p.cache.attention(qd, out=torch.empty_like(qd), window=21, sinks=1)
            for step in range(4):
                out.fill_(float("nan"))
                g.replay()
                torch.cuda.synchronize()
                o = out.cpu().numpy()
                eager, ref = p.decode(q, 20, 1)
                assert_close(o, ref, p.dtype, f"{kv} replay {step}")
                assert np.array_equal(o, eager)
                p.append([0, 1, 2], [step, step, step],
                         *(rng.standard_normal((3, H, d)).astype(p.dtype) for _ in range(2)))


def test_graphs_outlive_growth():
    """Two captured decode calls and a captured prefill of one cache, replayed by
    turns with eager calls, other windows and joins between, which take the
    contexts' places and outgrow the workspaces: each replay returns what its
    call did, and an order of rows not yet uploaded is refused under capture."""
    print("[case] window graphs outlive growth", flush=True)
    rng = np.random.default_rng(26)
    H, d, n_q = 4, 128, 40
    for kv in ("fp16", "kv4"):
        p = WPair(64, H, d, kv, 400)
        new = lambda n: [to_dev(rng.standard_normal((n, H, d)).astype(np.float16)) for _ in range(2)]
        for s, n in enumerate((700, 1500, 64)):
            p.cache.insert(s, np.arange(5000 * s, 5000 * s + n), *new(n))
        q, qp = new(3)[0], new(n_q)[0]
        ids, other = [2, 0, 1], [1, 0, 2]
        calls = [lambda o: p.cache.attention(q, out=o, window=600, sinks=2, seq_ids=ids),
                 lambda o: p.cache.attention(q, out=o, window=10 ** 9, sinks=0),
                 lambda o: p.cache.prefill(1, qp, out=o, window=1400, sinks=1)]
        outs = [torch.empty_like(x) for x in (q, q, qp)]
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            want, graphs = [], []
            for f, o in zip(calls, outs):
                f(o)
                want.append(o.clone())
            torch.cuda.synchronize()
            for f, o in zip(calls, outs):
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=stream):
                    f(o)
                    if f is calls[0]:
                        with pytest.raises(ChunkAttnError):
                            p.cache.attention(q, out=torch.empty_like(q), window=600, sinks=2, seq_ids=other)
                graphs.append(g)
            eager = [lambda: p.cache.attention(q, window=600, sinks=2, seq_ids=other),
                     lambda: (p.cache.attention(q, window=33), p.cache.attention(q, window=44, sinks=7)),
                     lambda: [p.cache.insert(10 + i, np.arange(10 ** 5 + 900 * i, 10 ** 5 + 900 * i + 800), *new(800))
                              for i in range(12)],
                     lambda: (p.cache.attention(torch.zeros(15, H, d, dtype=torch.float16, device="cuda"), window=500),
                              p.cache.prefill(1, torch.zeros(700, H, d, dtype=torch.float16, device="cuda"),
                                              window=1400)),
                     lambda: torch.full((1 << 22,), 0xFF, dtype=torch.uint8, device="cuda")]
            for step in eager:
                step()
                for _ in range(2):
                    for g, o, w in zip(graphs, outs, want):
                        o.fill_(float("nan"))
                        g.replay()
                        torch.cuda.synchronize()
                        assert torch.equal(o, w), kv


@pytest.mark.parametrize("kv", KINDS)
@pytest.mark.parametrize("c", [16, 64])
def test_far_strides(kv, c):
    """Slots and heads so far apart that offsets pass 32 bits: every call returns
    the very values that it returns over dense pools."""
    print(f"[case] far strides {kv} c={c}", flush=True)
    rng = np.random.default_rng(27)
    H, d, L = 2, 128, 30 * c + 5
    dt = torch.float32 if kv == "fp32" else torch.float16
    bits = 4 if kv == "kv4" else None
    near, far = (Cache(c, H, d, 40, dtype=dt, kv_bits=bits) for _ in range(2))
    # far: K of (slot s, head h) at byte s * 320 MB + h * 100 MB, V 50 MB behind
    mb = 1 << 20
    pool = torch.empty(40 * 320 * mb, dtype=torch.uint8, device="cuda")
    binding.ca_destroy(far.h)
    es = 1 if bits else near.k_pool.element_size()
    code = {"fp16": binding.CA_FP16, "fp32": binding.CA_FP32, "kv4": binding.CA_FP16_KV4}[kv]
    far.h = binding.ca_create(c, H, d, code, 40, pool.data_ptr(), pool.data_ptr() + 50 * mb,
                              slot_stride=320 * mb // es, head_stride=100 * mb // es)
    rows = [to_dev(rng.standard_normal((L, H, d))).to(dt) for _ in range(2)]
    own = [to_dev(rng.standard_normal((70, H, d))).to(dt) for _ in range(2)]
    q, qp = to_dev(rng.standard_normal((2, H, d))).to(dt), to_dev(rng.standard_normal((300, H, d))).to(dt)
    got = []
    for cache in (near, far):
        cache.insert(0, np.arange(L), *rows)
        cache.insert(1, np.concatenate([np.arange(L - 100), 10 ** 6 + np.arange(70)]),
                     *(torch.cat([r[:L - 100], o]) for r, o in zip(rows, own)))
        outs = [cache.attention(q, window=15 * c, sinks=3), cache.attention(q, window=10 ** 9)]
        if kv == "kv4":  # (the plain fp32 call may fold its partials in any order)
            outs.append(cache.attention(q))
        if kv != "fp32":
            outs += [cache.prefill(0, qp), cache.prefill(0, qp, window=13 * c, sinks=20), cache.prefill(1, qp[:7])]
        got.append([o.cpu() for o in outs])
        torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(*got)):
        assert torch.isfinite(a).all() and torch.equal(a, b), (i, (a - b).abs().max())
    near.close()
    far.close()


def test_refusals():
    c = Cache(64, 2, 64, 8)
    kv = torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda")
    c.insert(0, [1, 2, 3, 4], kv, kv)
    q = kv[:1].contiguous()
    for window, sinks in ((0, 0), (-1, 0), (4, -1)):
        with pytest.raises(ChunkAttnError):
            c.attention(q, window=window, sinks=sinks)
    with pytest.raises(ValueError):
        c.attention(q, sinks=4)
    with pytest.raises(ChunkAttnError):
        c.attention(q, window=4, seq_ids=[1])
    with pytest.raises(ChunkAttnError):
        c.attention(q, window=4, seq_ids=[0, 0])
    with pytest.raises(ChunkAttnError):
        c.attention(q, window=4, scale=-1.0)
    with pytest.raises(ValueError):
        c.attention(kv, window=4)
    c.close()
