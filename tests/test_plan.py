"""The decode plan of windowed calls and of 4-bit caches, on the CPU: its
coverage over random trees (plan_check.cpp, built with the sanitizers), the
entry points over a table-only cache, refusals."""
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2402_15220_amd import binding as B
from paper_2402_15220_amd.cache import Cache

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2402_15220_amd", "csrc")


def test_plan_covers_what_rows_see(tmp_path):
    exe = str(tmp_path / "plan_check")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", f"-I{CSRC}",
                        os.path.join(HERE, "plan_check.cpp")] +
                       [os.path.join(CSRC, f) for f in ("plan.cpp", "tables.cpp", "tree.cpp")] + ["-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr[-3000:]


@pytest.mark.parametrize("kv_bits", [None, 4])
def test_workspace_of_a_table_only_cache(kv_bits):
    c = Cache(16, 2, 64, 1000, table_only=True, kv_bits=kv_bits)
    for s in range(5):
        c.insert(s, np.concatenate([np.arange(200), 1000 + 300 * s + np.arange(20 * s + 1)]))
    assert B.ca_window_workspace_size(c.h, 1, 0) == 0          # the last token only: one piece a row
    whole = B.ca_window_workspace_size(c.h, 1 << 40, 0)
    assert whole > 0                                           # shared and private pieces
    if kv_bits == 4:
        assert B.ca_workspace_size(c.h) == whole
    assert not c.prepare(window=5, sinks=2)                    # nothing to upload
    assert not c.prepare()
    assert len(c.seq_order()) == 5
    c.append([0, 1], [7, 7])
    c.remove(3)
    assert len(c.seq_order()) == 4 and c.stats()["patches"] >= 0
    c.close()


def test_refusals():
    with pytest.raises(ValueError):
        Cache(64, 2, 64, 8, dtype=torch.float32, table_only=True, kv_bits=4)
    with pytest.raises(ValueError):
        Cache(64, 2, 64, 8, table_only=True, kv_bits=3)
    c = Cache(64, 2, 64, 8, table_only=True)
    for window, sinks in ((0, 0), (-5, 0), (3, -1)):
        with pytest.raises(B.ChunkAttnError):
            B.ca_window_workspace_size(c.h, window, sinks)
        with pytest.raises(B.ChunkAttnError):
            c.prepare(window=window, sinks=sinks)
    with pytest.raises(ValueError):
        c.prepare(sinks=1)
    with pytest.raises(B.ChunkAttnError):
        B.ca_attention_window(c.h, None, None, None, 4, 0, 0.0, None, 0)
    big = Cache(16385, 1, 64, 8, table_only=True)
    with pytest.raises(B.ChunkAttnError):
        big.prepare(window=5)
    big.close()
    with pytest.raises(B.ChunkAttnError):
        Cache(16385, 1, 64, 8, table_only=True, kv_bits=4)
    # 4-bit tiles: strides are bytes and a tile must fit them
    tile = 64 * 36
    with pytest.raises(B.ChunkAttnError):
        B.ca_create(64, 2, 64, B.CA_FP16_KV4, 4, 4096, 8192, slot_stride=2 * tile, head_stride=tile - 16)
    c.close()
