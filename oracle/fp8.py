"""Plain CPU oracle for the layer in 8 bits, its append, and the maps of a step.

TEST INFRASTRUCTURE ONLY (see ``oracle.paged_kv``).

Layer (bytes), one block after another::

    [2 (K, V)][num_kv_heads][block_size * head_dim] e4m3 codes
    [num_kv_heads][2 (K, V)]                        exponent + 127
    padding to a multiple of 128

    K tile: token r, dim j at (j // 16 * 16 + r) * 16 + j % 16
    V tile: token r, dim j at
        j // 64 * 1024 + r // 4 * 256 + j % 16 * 16 + j // 16 % 4 * 4 + r % 4

A tile's values are code * 2 ** (byte - 127). ``to_bf16_layer`` writes them, exactly,
into a layer of the bf16 format, so that attention over a layer in 8 bits is
``oracle.paged_kv``'s over that one.
"""
from __future__ import annotations

import numpy as np

BS = 16
E_MIN, E_MAX = -117, 119
NAN_CODE = 0x7F


def block_bytes(num_kv_heads: int, head_dim: int) -> int:
    return 2 * num_kv_heads * BS * head_dim + -(-2 * num_kv_heads // 128) * 128


def decode(codes: np.ndarray) -> np.ndarray:
    """e4m3 codes as fp64: sign, 4 bits of exponent (bias 7), 3 of mantissa; no
    infinities, NaN where the other seven bits are set."""
    c = np.asarray(codes, dtype=np.uint8).astype(np.int64)
    exp, man = (c >> 3) & 15, c & 7
    mag = np.where(exp > 0, (8 + man) * np.exp2(exp - 10.0), man * np.exp2(-9.0))
    mag = np.where((c & 127) == 127, np.nan, mag)
    return np.where(c & 128, -mag, mag)


def encode(x: np.ndarray) -> np.ndarray:
    """fp64 to the nearest e4m3 code, ties to even; past 448 the largest code."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    e = np.frexp(np.maximum(a, 2.0 ** -6))[1] - 1            # binade, at least 2^-6
    steps = np.minimum(np.rint(a / np.exp2(e - 3.0)), 16)    # 8 .. 16 in a normal binade
    up = steps == 16
    e, steps = np.where(up, e + 1, e), np.where(up, 8, steps)
    code = np.where(steps >= 8, ((e + 7) << 3) + (steps.astype(np.int64) - 8),
                    steps.astype(np.int64))
    code = np.minimum(code, 0x7E)
    code = np.where(np.isfinite(x), code, NAN_CODE)
    return np.where(np.signbit(x), code | 128, code).astype(np.uint8)


def exponent(amax) -> np.ndarray:
    """Least e with amax <= 448 * 2 ** e, within the exponents in use."""
    m, p = np.frexp(np.asarray(amax, dtype=np.float64))      # amax = m 2^p, m in [0.5, 1)
    e = p - 9 + (m > 0.875)                                  # 448 = 0.875 * 2^9
    return np.where(np.asarray(amax) > 0, np.clip(e, E_MIN, E_MAX), E_MIN).astype(np.int64)


def place(kind: int, r, j):
    """Where token r, dim j of a K (0) or V (1) tile lies."""
    r, j = np.asarray(r), np.asarray(j)
    if kind == 0:
        return (j // 16 * 16 + r) * 16 + j % 16
    return j // 64 * 1024 + r // 4 * 256 + j % 16 * 16 + j // 16 % 4 * 4 + r % 4


class Layer:
    """Views of a layer's bytes: ``codes`` [blocks, 2, heads, 16 * d], ``exps`` [blocks, heads, 2]."""

    def __init__(self, raw: np.ndarray, num_kv_heads: int, head_dim: int):
        self.raw = raw.reshape(-1, block_bytes(num_kv_heads, head_dim))
        n, size = len(self.raw), BS * head_dim
        at = 2 * num_kv_heads * size
        self.codes = self.raw[:, :at].reshape(n, 2, num_kv_heads, size)
        self.exps = self.raw[:, at:at + 2 * num_kv_heads].reshape(n, num_kv_heads, 2)
        # reshape of a sliced row may copy: write through these instead
        self._at, self._size, self.heads, self.dim = at, size, num_kv_heads, head_dim

    def tile(self, b: int, kind: int, g: int) -> np.ndarray:
        o = (kind * self.heads + g) * self._size
        return self.raw[b, o:o + self._size]

    def exp(self, b: int, kind: int, g: int) -> int:
        return int(self.raw[b, self._at + 2 * g + kind])

    def set_exp(self, b: int, kind: int, g: int, byte: int) -> None:
        self.raw[b, self._at + 2 * g + kind] = byte

    def values(self, b: int, kind: int, g: int) -> np.ndarray:
        """[16, d] in fp64."""
        t = decode(self.tile(b, kind, g)) * np.exp2(self.exp(b, kind, g) - 127.0)
        return t[place(kind, np.arange(BS)[:, None], np.arange(self.dim)[None, :])]


def append(raw: np.ndarray, k_new: np.ndarray, v_new: np.ndarray, slot_mapping, *,
           num_kv_heads: int, head_dim: int) -> np.ndarray:
    """Copy of the layer's bytes with the new rows (fp64 [T, heads, d]) written. Tokens of
    one block stand together in the list."""
    out = np.array(raw, copy=True)
    lay = Layer(out, num_kv_heads, head_dim)
    cap = len(lay.raw) * BS
    slots = [int(s) if 0 <= int(s) < cap else -1 for s in slot_mapping]
    j = np.arange(head_dim)
    t = 0
    while t < len(slots):
        if slots[t] < 0:
            t += 1
            continue
        end = t
        while end < len(slots) and slots[end] >= 0 and slots[end] // BS == slots[t] // BS:
            end += 1
        b, rows = slots[t] // BS, [s % BS for s in slots[t:end]]
        for kind, new in ((0, k_new), (1, v_new)):
            for g in range(num_kv_heads):
                x = np.asarray(new[t:end, g], dtype=np.float64)
                fin = np.where(np.isfinite(x), np.abs(x), 0.0)
                e = int(exponent(fin.max()))
                tile = lay.tile(b, kind, g)
                if 0 not in rows:
                    old = min(max(lay.exp(b, kind, g) - 127, E_MIN), E_MAX)
                    if e > old:
                        c = decode(tile)
                        tile[:] = np.where(np.isnan(c), tile, encode(c * np.exp2(float(old - e))))
                    e = max(e, old)
                lay.set_exp(b, kind, g, e + 127)
                for i, r in enumerate(rows):
                    tile[place(kind, r, j)] = encode(x[i] * np.exp2(float(-e)))
        t = end
    return out


def to_bf16_layer(raw: np.ndarray, num_kv_heads: int, head_dim: int) -> np.ndarray:
    """The layer's values as bf16 bit patterns (uint16) in the bf16 layout; exact. Tiles whose
    exponent is none in use become NaN."""
    lay = Layer(raw, num_kv_heads, head_dim)
    n = len(lay.raw)
    exps = lay.exps.transpose(0, 2, 1)[..., None] - 127.0
    exps = np.where((exps < E_MIN) | (exps > E_MAX), np.nan, exps)   # of a block never begun
    codes = decode(lay.codes) * np.exp2(exps)
    r, j = np.arange(BS)[:, None], np.arange(head_dim)[None, :]
    out = np.empty((n, 2, num_kv_heads, BS * head_dim), np.float64)
    to = ((j // 8 * BS + r) * 8 + j % 8, j * BS + r)
    for kind in range(2):
        out[:, kind][..., to[kind]] = codes[:, kind][..., place(kind, r, j)]
    f = out.astype(np.float32)
    assert np.array_equal(f, out, equal_nan=True)
    bits = f.reshape(-1).view(np.uint32)
    assert not (bits[np.isfinite(f.reshape(-1))] & 0xFFFF).any()
    return (bits >> 16).astype(np.uint16)


def from_bf16_layer(kv_raw: np.ndarray, num_kv_heads: int, head_dim: int) -> np.ndarray:
    """Bytes of a layer in 8 bits from bf16 bit patterns in the bf16 layout, each tile
    with the least exponent for its finite values; NaN stays NaN."""
    x = (np.asarray(kv_raw, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    x = x.reshape(-1, 2, num_kv_heads, BS * head_dim)
    out = np.zeros((len(x), block_bytes(num_kv_heads, head_dim)), np.uint8)
    e = exponent(np.where(np.isfinite(x), np.abs(x), 0.0).max(-1))          # [n, 2, heads]
    codes = encode(x * np.exp2(-e[..., None].astype(np.float64)))
    r, j = np.arange(BS)[:, None], np.arange(head_dim)[None, :]
    at = ((j // 8 * BS + r) * 8 + j % 8, j * BS + r)
    tiles = np.empty_like(codes)
    for kind in range(2):
        tiles[:, kind][..., place(kind, r, j)] = codes[:, kind][..., at[kind]]
    size = 2 * num_kv_heads * BS * head_dim
    out[:, :size] = tiles.reshape(len(x), -1)
    out[:, size:size + 2 * num_kv_heads] = (e + 127).transpose(0, 2, 1).reshape(len(x), -1)
    return out.reshape(-1)


def step_map(cached, new, free_ids, block_table, max_tokens: int):
    """Token by token: (seq_lens, cu, slots, positions, used, table)."""
    table = np.array(block_table, dtype=np.int64, copy=True)
    S, MB = table.shape
    free = [int(i) for i in free_ids]
    lens, cu, slots, positions, taken = [], [0], [], [], 0
    for s in range(S):
        pos = max(int(cached[s]), 0)
        for _ in range(max(int(new[s]), 0)):
            if pos >= MB * BS or len(slots) == max_tokens:
                break
            if pos % BS == 0:
                table[s, pos // BS] = free[taken] if taken < len(free) else -1
                taken += 1
            block = table[s, pos // BS]
            slots.append(int(block) * BS + pos % BS if block >= 0 else -1)
            positions.append(pos)
            pos += 1
        lens.append(pos)
        cu.append(len(slots))
    total = len(slots)
    slots += [-1] * (max_tokens - total)
    positions += [0] * (max_tokens - total)
    return lens, cu, slots, positions, [total, taken], table
