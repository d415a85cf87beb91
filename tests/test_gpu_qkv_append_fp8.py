"""Norm, rotation and cache write into a layer in 8 bits, against the oracle: exponents, v and
what other slots hold byte for byte, k's codes within half a step of e4m3 (2^-4 of a value, 2^-10
below its normal range) and fp32's error, as in ``test_gpu_qkv_append``."""
import numpy as np
import pytest
import torch

import paper_2608_23658_amd.kvattn as K
from oracle import fp8
from tests.gpu_helpers import require_gpu, say
from tests.test_gpu_qkv_append import FP32_ERROR, Rows, assert_rounded, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def in_blocks(T, start, seed=0, spare=3):
    """A chunk's slots from slot ``start`` of a block on, blocks in any order."""
    nb = (T + start) // 16 + spare
    perm = np.random.default_rng(seed).permutation(nb)
    t = np.arange(start, start + T)
    return nb, perm[t // 16] * 16 + t % 16


def one_a_block(T, seed=0):
    r = np.random.default_rng(seed)
    nb = T + 7
    return nb, r.permutation(nb)[:T] * 16 + r.integers(0, 16, T)


def layer_of(nb, hkv, d, seed=0):
    r = np.random.default_rng(seed)
    raw = r.integers(0, 256, (nb, fp8.block_bytes(hkv, d)), dtype=np.uint8)
    at = 2 * hkv * 16 * d
    raw[:, at:at + 2 * hkv] = r.integers(112, 124, (nb, 2 * hkv))
    return raw.reshape(-1)


def check(r, what, seed=0):
    say("qkv append fp8", what, r.T, r.hq, r.hkv, r.d, r.dtype)
    raw = layer_of(r.nb, r.hkv, r.d, seed)
    r.layer = torch.from_numpy(raw.copy()).cuda()
    out = r.call(K.qkv_append_fp8)
    torch.cuda.synchronize()
    ref, size = r.expected("q")
    assert_rounded(f64(out), ref, size, r.dtype, what + " q")
    ref, size = r.expected("k")
    want = fp8.append(raw, ref, f64(r.v), r.slots, num_kv_heads=r.hkv, head_dim=r.d)
    got, want = fp8.Layer(r.layer.cpu().numpy(), r.hkv, r.d), fp8.Layer(want, r.hkv, r.d)
    end = got._at + 2 * r.hkv
    assert np.array_equal(got.raw[:, got._at:], want.raw[:, want._at:]), "exponents, or bytes past"
    new = np.zeros((r.nb, 2, r.hkv, 16 * r.d), bool)
    j = np.arange(r.d)
    for t, s in enumerate(r.slots):
        if not 0 <= s < r.nb * 16:
            continue
        b, at = s // 16, fp8.place(0, s % 16, j)
        new[b, 0][:, at] = True
        scale = np.exp2(got.exps[b, :, 0].astype(float) - 127.0)[:, None]
        x, m = ref[t] / scale, size[t] / scale
        y = fp8.decode(got.codes[b, 0][:, at])
        nan = ~np.isfinite(x)                # infinities become NaN too
        assert np.array_equal(np.isnan(y), nan)
        x, m = np.where(nan, 0, x), np.where(nan, 0, m)
        tol = FP32_ERROR * m * (1 + 2.0 ** -4) + np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10)
        assert (np.abs(y - x) <= tol)[~nan].all(), (what, t)
    a, b = got.codes.copy(), want.codes.copy()
    for c in (a, b):
        c[(c & 127) == 127] = 127            # one code of NaN is as good as the other
    assert np.array_equal(a[~new], b[~new]), what
    assert end <= got.raw.shape[1]


SHAPES = [("bf16", 8, 2, 128), ("bf16", 3, 1, 64), ("f32", 4, 2, 128), ("f32", 6, 3, 64)]


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("share", [None, 1, 2, 4])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotations(dtype, hq, hkv, d, share, interleaved):
    """No rotation, and all, half and a quarter (32 dims at least) of the dims."""
    nb, slots = in_blocks(37, 3)
    check(Rows(37, hq, hkv, d, dtype, rot=share and max(32, d // share), interleaved=interleaved,
               nb=nb, slots=slots), f"share {share}")


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("T,start", [(1, 0), (1, 9), (15, 1), (16, 0), (17, 15), (300, 5)])
def test_chunks(dtype, hq, hkv, d, T, start):
    nb, slots = in_blocks(T, start, T)
    check(Rows(T, hq, hkv, d, dtype, rot=d, nb=nb, slots=slots, seed=T, fused=T % 2 == 0),
          f"chunk from {start}")


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES[:2])
@pytest.mark.parametrize("T", [3, 200, 700, 2100])
def test_one_token_a_block(dtype, hq, hkv, d, T):
    """Every size of window; padding and slots outside among them."""
    nb, slots = one_a_block(T, T)
    slots[0], slots[1] = -1, nb * 16
    check(Rows(T, hq if T < 1000 else 2, hkv, d, dtype, rot=32, nb=nb, slots=slots, seed=T),
          "one a block")


@pytest.mark.parametrize("norm", [(False, False), (True, False), (False, True)])
def test_norms_apart(norm):
    nb, slots = in_blocks(21, 0)
    check(Rows(21, 4, 4, 64, "bf16", norm=norm, rot=64, nb=nb, slots=slots), f"norm {norm}")


@pytest.mark.parametrize("dtype,d,rot", [("bf16", 128, 128), ("bf16", 64, 32), ("f32", 128, 128)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_axes(dtype, d, rot, interleaved):
    nb, slots = in_blocks(40, 2)
    check(Rows(40, 3, 2, d, dtype, rot=rot, axes=3, sections=[3, 0, rot // 2 - 3],
               interleaved=interleaved, nb=nb, slots=slots), "axes")


def test_special_values():
    """NaN and infinities do not count for the exponent; a position outside the table gives
    NaN."""
    nb, slots = in_blocks(20, 0)
    r = Rows(20, 2, 2, 64, "f32", norm=(False, False), rot=32, max_pos=50, nb=nb, slots=slots)
    r.k[1, 0, 40], r.k[2, 1, 41], r.v[3, 0, 5] = float("nan"), float("inf"), float("-inf")
    r.k[4] = 0
    r.pos[7] = 50
    check(r, "special")


def test_into_blocks_that_hold_larger_and_smaller_numbers():
    """Tokens added to a block: its exponent stays or is raised, the others' codes follow."""
    r = Rows(24, 2, 2, 128, "bf16", rot=128, nb=30, slots=np.arange(24) * 16 + 3)
    for big in (1.0, 2.0 ** 9, 2.0 ** -9):
        r.wk = (torch.ones(128) * big).to(torch.bfloat16).cuda()
        check(r, f"size {big}")
