"""Plain fp64 CPU oracle for attention whose scores are capped, biased by distance or cut to
a window.

TEST INFRASTRUCTURE ONLY (see ``oracle.paged_kv``).

The row at position ``p`` of query head ``h`` gives key ``t``::

    a = scale * q . k
    a = softcap * tanh(a / softcap)        if softcap
    a = a + slopes[h] * (t - p)            if slopes
    seen: max(0, p - window + 1) <= t <= p     (no window: 0 <= t <= p)
    out = sum_t softmax_t(a) v

Blocks that no row of a sequence sees are not looked at, nor are tokens before the first
that any row sees.
"""
from __future__ import annotations

import numpy as np

from .paged_kv import gather_kv, storage_to_f64


def scores(q, k, rows, keys, *, scale, softcap=0.0, slope=0.0, window=0):
    """[n, keys] of one head's rows ``q`` at positions ``rows``; -inf where not seen."""
    a = scale * (q @ k.T)
    if softcap:
        a = softcap * np.tanh(a / softcap)
    ago = rows[:, None] - keys[None, :]
    a = a - slope * ago
    gone = (ago < 0) | ((ago >= window) if window else False)
    a[gone] = -np.inf
    return a


def scored_attention(q_raw, kv_raw, block_table, seq_lens, cu_seqlens_q, *, dtype, num_q_heads,
                     num_kv_heads, head_dim, scale, softcap=0.0, slopes=None, window=0,
                     block_size=16):
    """fp64 ([T, Hq, d] out, the same of sum p |v|). A sequence of length 0 gives zeros; ids
    outside the layer contribute nothing."""
    T = int(cu_seqlens_q[-1])
    q = storage_to_f64(np.asarray(q_raw).reshape(T, num_q_heads, head_dim), dtype)
    out, weight = np.zeros_like(q), np.zeros_like(q)
    group = num_q_heads // num_kv_heads
    esz = 2 if dtype == "bf16" else 4
    num_blocks = len(np.asarray(kv_raw).reshape(-1)) // (2 * num_kv_heads * block_size * head_dim)
    assert esz in (2, 4)
    for s, L in enumerate(int(x) for x in seq_lens):
        r0, r1 = int(cu_seqlens_q[s]), int(cu_seqlens_q[s + 1])
        n = r1 - r0
        if n == 0 or L == 0:
            continue
        first = max(0, L - n - window + 1) if window else 0
        base = first // block_size
        ids = np.asarray(block_table[s][base:-(-L // block_size)])
        there = (ids >= 0) & (ids < num_blocks)
        k, v = gather_kv(kv_raw, dtype, np.where(there, ids, 0), L - base * block_size,
                         num_kv_heads, block_size, head_dim)
        keys = np.arange(base * block_size, L)
        live = there[(keys - base * block_size) // block_size] & (keys >= first)
        k, v, keys = k[live], v[live], keys[live]
        rows = np.arange(L - n, L)
        for h in range(num_q_heads):
            a = scores(q[r0:r1, h], k[:, h // group], rows, keys, scale=scale, softcap=softcap,
                       slope=0.0 if slopes is None else float(slopes[h]), window=window)
            top = a.max(1, keepdims=True, initial=-np.inf)
            w = np.exp(a - np.where(np.isfinite(top), top, 0))
            z = w.sum(1, keepdims=True)
            z[z == 0] = 1
            vh = v[:, h // group]
            out[r0:r1, h], weight[r0:r1, h] = (w @ vh) / z, (w @ np.abs(vh)) / z
    return out, weight
