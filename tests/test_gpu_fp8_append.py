"""Writing rows into a layer in 8 bits: byte for byte against the oracle."""
import numpy as np
import pytest
import torch

import paper_2608_23658_amd.kvattn as K
from oracle import fp8
from tests.gpu_helpers import require_gpu, say

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _layer(nb, hkv, d, seed):
    r = np.random.default_rng(seed)
    raw = r.integers(0, 256, (nb, fp8.block_bytes(hkv, d)), dtype=np.uint8)
    at = 2 * hkv * 16 * d
    raw[:, at:at + 2 * hkv] = r.integers(115, 125, (nb, 2 * hkv))
    return raw.reshape(-1)


def _rows(T, hkv, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    size = torch.exp2(torch.randint(-6, 6, (T, hkv, 1), generator=g).float())
    return [(torch.randn(T, hkv, d, generator=g) * size).to(DT[dtype]) for _ in range(2)]


def _check(raw, k, v, slots, hkv, d, stream=None):
    slots = np.asarray(slots, np.int32)
    nb = len(raw) // fp8.block_bytes(hkv, d)
    dl = torch.from_numpy(raw.copy()).cuda()
    K.kv_append_fp8(k.cuda(), v.cuda(), torch.from_numpy(slots).cuda(), dl, nb)
    torch.cuda.synchronize()
    got = dl.cpu().numpy()
    want = fp8.append(raw, k.double().numpy(), v.double().numpy(), slots, num_kv_heads=hkv,
                      head_dim=d)
    # one code of NaN is as good as the other
    size = 2 * hkv * 16 * d

    def parts(x):
        x = x.reshape(nb, -1)
        c = x[:, :size].copy()
        c[(c & 127) == 127] = 127
        return c, x[:, size:]
    (gc, ge), (wc, we) = parts(got), parts(want)
    assert np.array_equal(ge, we), "exponents, or bytes past them"
    bad = np.argwhere(gc != wc)
    assert not len(bad), (len(bad), bad[:3], fp8.decode(gc[tuple(bad[0])]), fp8.decode(wc[tuple(bad[0])]))
    return got


SHAPES = [("bf16", 8, 128), ("bf16", 3, 64), ("f32", 2, 128), ("f32", 1, 64), ("bf16", 65, 64)]


@pytest.mark.parametrize("dtype,hkv,d", SHAPES)
@pytest.mark.parametrize("T,start", [(1, 0), (1, 7), (16, 0), (15, 1), (17, 15), (300, 5)])
def test_chunk(dtype, hkv, d, T, start):
    say("append fp8 chunk", dtype, hkv, d, T, start)
    nb = (T + start) // 16 + 3
    perm = np.random.default_rng(T).permutation(nb)
    t = np.arange(start, start + T)
    k, v = _rows(T, hkv, d, dtype, T + d)
    _check(_layer(nb, hkv, d, T), k, v, perm[t // 16] * 16 + t % 16, hkv, d)


@pytest.mark.parametrize("dtype,hkv,d", SHAPES[:3])
@pytest.mark.parametrize("T", [5, 256, 1500, 2200])
def test_scattered(dtype, hkv, d, T):
    """One token per block at any place in it, with padding and slots past the layer."""
    say("append fp8 scattered", dtype, hkv, d, T)
    hkv = min(hkv, 2) if T > 1000 else hkv
    r = np.random.default_rng(T)
    nb = T + 9
    slots = r.permutation(nb)[:T] * 16 + r.integers(0, 16, T)
    slots[1] = -1
    slots[3] = nb * 16
    slots[r.random(T) < 0.1] = -7
    k, v = _rows(T, hkv, d, dtype, T)
    _check(_layer(nb, hkv, d, T), k, v, slots, hkv, d)


@pytest.mark.parametrize("T", [400, 900, 2600])
def test_runs_of_every_length(T):
    """Ragged pieces of sequences, in pieces of 1 to 40 tokens from any slot on; windows
    of the list begin anywhere in them."""
    say("append fp8 ragged", T)
    r = np.random.default_rng(T)
    nb, slots, free = 2 * T, [], iter(r.permutation(2 * T))
    while len(slots) < T:
        n, at = int(r.integers(1, 41)), int(r.integers(0, 16))
        blocks = [next(free) for _ in range((at + n + 15) // 16)]
        piece = [blocks[(at + i) // 16] * 16 + (at + i) % 16 for i in range(n)]
        if r.random() < 0.3:       # any order inside a block
            piece = [s for b in blocks for s in r.permutation([p for p in piece if p // 16 == b])]
        slots += piece + [-1] * int(r.integers(0, 2))
    slots = slots[:T]
    k, v = _rows(T, 2, 64, "bf16", T)
    _check(_layer(nb, 2, 64, T), k, v, slots, 2, 64)


def test_token_by_token_raises_scales():
    """A block filled one token a call, each larger than all before by up to 2^40:
    codes of the early ones go through the subnormals to zero."""
    say("append fp8 token by token")
    hkv, d = 2, 128
    raw = _layer(2, hkv, d, 3)
    g = torch.Generator().manual_seed(1)
    for i in range(16):
        f = 2.0 ** (i if i < 12 else 10 * (i - 10))
        k, v = ((torch.randn(1, hkv, d, generator=g) * f).to(torch.bfloat16) for _ in range(2))
        raw = _check(raw, k, v, [16 + i], hkv, d)


def test_special_values():
    say("append fp8 special values")
    hkv, d = 1, 64
    for dtype in ("bf16", "f32"):
        k, v = _rows(6, hkv, d, dtype, 9)
        k[0, 0, 3], k[1, 0, 5], k[2, 0, 7] = float("inf"), float("nan"), -float("inf")
        v[:] = 0.0
        v[1, 0, 1] = -0.0
        v[4] = float("nan")
        _check(_layer(3, hkv, d, 4), k, v, [16, 17, 18, 40, 41, 5], hkv, d)
        big, tiny = _rows(2, hkv, d, dtype, 10)
        big = (big.double() * 1e38).to(DT[dtype])
        tiny = (tiny.double() * 1e-38).to(DT[dtype])
        _check(_layer(3, hkv, d, 4), big, tiny, [0, 1], hkv, d)
        _check(_layer(3, hkv, d, 4), tiny, big, [20, 21], hkv, d)
        # a value on the border of two exponents, and one step past it
        edge = torch.full((2, hkv, d), 448.0)
        edge[1] = 450.0 if dtype == "bf16" else 448.00003
        e = edge.to(DT[dtype])
        _check(_layer(3, hkv, d, 4), e[:1], e[1:], [0], hkv, d)


def test_nothing_and_all_padding():
    say("append fp8 nothing")
    hkv, d = 2, 64
    raw = _layer(2, hkv, d, 1)
    e = torch.empty(0, hkv, d, dtype=torch.bfloat16)
    assert np.array_equal(_check(raw, e, e, [], hkv, d), raw)
    k, v = _rows(5, hkv, d, "bf16", 1)
    assert np.array_equal(_check(raw, k, v, [-1] * 5, hkv, d), raw)


def test_repeated_slots_stay_inside_their_block():
    """A slot named twice is the caller's mistake: its block's contents are
    unspecified, and no other block changes."""
    say("append fp8 repeated slots")
    hkv, d, nb = 2, 64, 4
    raw = _layer(nb, hkv, d, 6)
    k, v = _rows(40, hkv, d, "bf16", 6)
    slots = np.array([16 + i % 3 for i in range(40)], np.int32)
    dl = torch.from_numpy(raw.copy()).cuda()
    K.kv_append_fp8(k.cuda(), v.cuda(), torch.from_numpy(slots).cuda(), dl, nb)
    got = dl.cpu().numpy().reshape(nb, -1)
    assert np.array_equal(np.delete(got, 1, 0), np.delete(raw.reshape(nb, -1), 1, 0))
