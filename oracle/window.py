"""Attention with a sliding window and sinks over the tree, in float64.

Test infrastructure only (see the package docstring).

The query at position p of a sequence sees the positions j <= p with
j < sinks or j > p - window. ``values`` maps the stored rows to what they
stand for (``kv4_values`` for a cache held in 4 bits).
"""
from __future__ import annotations

import numpy as np

from .attention import _softmax_attend


def visible(p, window, sinks):
    """Positions the query at position p sees."""
    j = np.arange(p + 1)
    return j if window is None else j[(j < sinks) | (j > p - window)]


def _path(tree, sid, values):
    nodes = tree.path(sid)
    k = np.concatenate([n.k for n in nodes], axis=0)
    v = np.concatenate([n.v for n in nodes], axis=0)
    return (values(k), values(v)) if values else (k.astype(np.float64), v.astype(np.float64))


def window_attention(tree, row_seq, q, scale, window, sinks=0, values=None):
    """o of every row (tree row order), float64 [B, H, d]."""
    out = np.empty(q.shape, np.float64)
    for r, sid in enumerate(row_seq):
        k, v = _path(tree, int(sid), values)
        j = visible(k.shape[0] - 1, window, sinks)
        out[r] = _softmax_attend(q[r].astype(np.float64), k[j], v[j], scale)
    return out


def window_prefill(tree, sid, q, scale, window, sinks=0, values=None):
    """o of the last q.shape[0] tokens of sequence sid, float64."""
    k, v = _path(tree, sid, values)
    out = np.empty(q.shape, np.float64)
    for i in range(q.shape[0]):
        j = visible(k.shape[0] - q.shape[0] + i, window, sinks)
        out[i] = _softmax_attend(q[i].astype(np.float64), k[j], v[j], scale)
    return out
