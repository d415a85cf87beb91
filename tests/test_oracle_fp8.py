"""The oracle of the layer in 8 bits: its rounding against torch's, its layout
against the documented offsets, its append against what the words say, and its step maps
against vectorised arithmetic."""
import numpy as np
import pytest
import torch

from oracle import fp8


def test_codes_decode_as_torch_does():
    c = np.arange(256, dtype=np.uint8)
    t = torch.from_numpy(c).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(fp8.decode(c), t, equal_nan=True)


def test_encode_rounds_to_nearest_even():
    vals = fp8.decode(np.arange(127, dtype=np.uint8))
    mids = (vals[1:] + vals[:-1]) / 2
    rng = np.random.default_rng(1)
    x = np.concatenate([vals, mids, np.nextafter(mids, 0), np.nextafter(mids, 1e9),
                        rng.normal(size=4000) * np.exp2(rng.integers(-12, 8, 4000))])
    x = np.concatenate([x, -x])
    x = x[np.abs(x) <= 448]
    got = fp8.decode(fp8.encode(x))
    # brute force: the nearest code, the even one of two
    d = np.abs(np.abs(x)[:, None] - vals[None, :])
    best = d.min(1, keepdims=True)
    pick = np.where(d == best, np.arange(127)[None, :] % 2, 2).argmin(1)
    assert np.array_equal(np.abs(got), vals[pick])
    assert np.array_equal(np.signbit(got), np.signbit(x))
    assert (fp8.encode([500.0, -1e30, np.nan, np.inf]) == [0x7E, 0xFE, 0x7F, 0x7F]).all()


def test_exponent_is_the_least_that_holds():
    for a in [1e-30, 0.1, 448.0, 448.0000001, 447.9, 896.0, 897.0, 1.0, 1e30]:
        e = int(fp8.exponent(a))
        assert a <= 448 * 2.0 ** e
        assert e == fp8.E_MIN or a > 448 * 2.0 ** (e - 1)
    assert fp8.exponent(0.0) == fp8.E_MIN
    assert fp8.exponent(3e38) == fp8.E_MAX


@pytest.mark.parametrize("d", [64, 128])
def test_places_cover_a_tile_once(d):
    r, j = np.arange(16)[:, None], np.arange(d)[None, :]
    for kind in range(2):
        assert sorted(fp8.place(kind, r, j).ravel()) == list(range(16 * d))
    assert fp8.place(0, 3, 37) == (2 * 16 + 3) * 16 + 5
    assert fp8.place(1, 6, 37) == 1 * 256 + 5 * 16 + 2 * 4 + 2


def test_layers_of_both_formats_agree():
    rng = np.random.default_rng(5)
    hkv, d, n = 2, 64, 3
    raw = rng.integers(0, 256, (n, fp8.block_bytes(hkv, d)), dtype=np.uint8)
    at = 2 * hkv * 16 * d
    raw[:, at:at + 2 * hkv] = rng.integers(10, 247, (n, 2 * hkv))
    bf = fp8.to_bf16_layer(raw.reshape(-1), hkv, d).reshape(n, 2, hkv, 16 * d)
    f = (bf.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    lay = fp8.Layer(raw.reshape(-1), hkv, d)
    for b, g, r, j in [(0, 0, 0, 0), (1, 1, 5, 17), (2, 0, 15, 63), (1, 0, 9, 40)]:
        assert f[b, 0, g, (j // 8 * 16 + r) * 8 + j % 8] == lay.values(b, 0, g)[r, j] or \
            np.isnan(lay.values(b, 0, g)[r, j])
        assert f[b, 1, g, j * 16 + r] == lay.values(b, 1, g)[r, j] or \
            np.isnan(lay.values(b, 1, g)[r, j])
    back = fp8.from_bf16_layer(bf.reshape(-1), hkv, d)
    assert np.array_equal(fp8.to_bf16_layer(back, hkv, d)[f.reshape(-1) == f.reshape(-1)],
                          bf.reshape(-1)[f.reshape(-1) == f.reshape(-1)])


def test_append_scales_a_block_anew():
    hkv, d = 1, 64
    raw = np.zeros(2 * fp8.block_bytes(hkv, d), np.uint8)
    x = np.zeros((3, hkv, d))
    x[0], x[1], x[2] = 1.0, 300.0, 0.25
    a = fp8.append(raw, x[:1], x[:1], [16], num_kv_heads=hkv, head_dim=d)
    lay = fp8.Layer(a, hkv, d)
    assert lay.exp(1, 0, 0) == 127 - 8 and (lay.values(1, 0, 0)[0] == 1.0).all()
    b = fp8.append(a, x[1:], x[1:], [17, 18], num_kv_heads=hkv, head_dim=d)
    lay = fp8.Layer(b, hkv, d)
    assert lay.exp(1, 1, 0) == 127
    assert [lay.values(1, 1, 0)[r, 7] for r in range(3)] == [1.0, 288.0, 0.25]
    c = fp8.append(b, x[2:], x[2:], [16], num_kv_heads=hkv, head_dim=d)   # begins anew
    assert fp8.Layer(c, hkv, d).exp(1, 0, 0) == 127 - 10
    assert (a[:fp8.block_bytes(hkv, d)] == raw[:fp8.block_bytes(hkv, d)]).all()
    assert (fp8.append(raw, x, x, [-1, 32, 1 << 30], num_kv_heads=hkv, head_dim=d) == raw).all()


def test_step_map_by_hand():
    table = np.full((3, 4), -1)
    table[0, :2], table[2, :1] = [7, 8], [9]
    lens, cu, slots, pos, used, out = fp8.step_map([17, 0, 16], [1, 18, 40], [3, 4, 5], table, 24)
    assert lens == [18, 18, 21] and cu == [0, 1, 19, 24] and used == [24, 3]
    assert slots[:3] == [8 * 16 + 1, 48, 49] and slots[17:20] == [64, 65, 80]
    assert pos[0] == 17 and pos[19] == 16
    assert out.tolist() == [[7, 8, -1, -1], [3, 4, -1, -1], [9, 5, -1, -1]]


def test_scaling_anew_is_exact_down_to_the_normal_range():
    """A block's code c 2^old under the exponent of larger values: exact where it is at least
    2^-6 of the new power of two, which is less than 2^-13.8 of the largest, and not 2^-14 of
    it: 225 takes exponent 0, and 2^-13.9 of that is rounded."""
    codes = fp8.decode(np.arange(127, dtype=np.uint8))
    for amax in (225.0, 300.0, 448.0, 449.0, 1e5):
        e = int(fp8.exponent(amax))
        assert 2.0 ** (e - 6) < 2.0 ** -13.8 * amax
        for old in range(e - 24, e):
            v = codes * 2.0 ** old
            got = fp8.decode(fp8.encode(v * 2.0 ** -e)) * 2.0 ** e
            normal = v >= 2.0 ** (e - 6)
            assert np.array_equal(got[normal], v[normal])
    raw = np.zeros(fp8.block_bytes(1, 64), np.uint8)
    small, large = np.full((1, 1, 64), 0.0146484375), np.full((1, 1, 64), 225.0)
    assert 2.0 ** -14 < 0.0146484375 / 225 < 2.0 ** -13.8
    for slot, x, seen in ((0, small, 0.0146484375), (1, large, 0.015625)):
        raw = fp8.append(raw, x, x, [slot], num_kv_heads=1, head_dim=64)
        assert (fp8.Layer(raw, 1, 64).values(0, 0, 0)[0] == seen).all()
