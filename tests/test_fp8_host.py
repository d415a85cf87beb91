"""What the calls on a layer in 8 bits and the step maps refuse, before anything is
launched: the C ABI's checks with addresses that are never touched, and the
binding's with CPU tensors."""
import pytest
import torch

import paper_2608_23658_amd.kvattn as K
from oracle import fp8

A = 1 << 20


@pytest.fixture(scope="module")
def L():
    return K.lib()


def test_block_bytes(L):
    for hkv in (1, 3, 8, 64, 65, 65535):
        for d in (64, 128):
            assert K.fp8_block_bytes(hkv, d) == fp8.block_bytes(hkv, d)
            assert K.fp8_block_bytes(hkv, d) % 128 == 0
    assert K.fp8_block_bytes(0, 128) == K.fp8_block_bytes(8, 96) == K.fp8_block_bytes(-1, 64) == 0
    assert K.fp8_block_bytes(65536, 64) == 0


def _decode(L, **kw):
    a = dict(q=A, kv=A, nb=100, bt=A, sl=A, out=A, B=4, hq=32, hkv=8, d=128, bs=16, mb=10,
             msl=160, scale=0.1, dt=K.KV_BF16, ws=A, wsb=1 << 30)
    a.update(kw)
    return L.kvattn_decode_fp8(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(d=96), K.KV_ERR_UNSUPPORTED), (dict(d=64, dt=K.KV_F32), K.KV_ERR_UNSUPPORTED),
    (dict(hq=24), K.KV_ERR_UNSUPPORTED), (dict(hq=30), K.KV_ERR_INVALID),
    (dict(bs=32), K.KV_ERR_UNSUPPORTED), (dict(dt=7), K.KV_ERR_INVALID),
    (dict(msl=161), K.KV_ERR_INVALID), (dict(nb=0), K.KV_ERR_INVALID),
    (dict(q=A + 8), K.KV_ERR_INVALID), (dict(kv=A + 4), K.KV_ERR_INVALID),
    (dict(out=0), K.KV_ERR_INVALID), (dict(wsb=100), K.KV_ERR_INVALID),
    (dict(scale=float("nan")), K.KV_ERR_INVALID), (dict(B=-1), K.KV_ERR_INVALID),
])
def test_decode_refuses(L, kw, code):
    assert _decode(L, **kw) == code
    assert K.last_error().startswith("kvattn_decode_fp8")


def _prefill(L, **kw):
    a = dict(q=A, kv=A, nb=100, bt=A, sl=A, cu=A, out=A, B=2, T=100, budget=128, hq=32, hkv=8,
             d=128, bs=16, mb=10, msl=160, scale=0.1, dt=K.KV_BF16, ws=A, wsb=1 << 20)
    a.update(kw)
    return L.kvattn_prefill_chunk_fp8(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dt=K.KV_F32), K.KV_ERR_UNSUPPORTED), (dict(d=64), K.KV_ERR_UNSUPPORTED),
    (dict(hq=128), K.KV_ERR_UNSUPPORTED), (dict(T=200), K.KV_ERR_INVALID),
    (dict(cu=0), K.KV_ERR_INVALID), (dict(wsb=16), K.KV_ERR_INVALID),
    (dict(msl=1000), K.KV_ERR_INVALID), (dict(nb=0), K.KV_ERR_INVALID),
    (dict(kv=A + 8), K.KV_ERR_INVALID), (dict(scale=float("inf")), K.KV_ERR_INVALID),
    (dict(scale=0.0), K.KV_ERR_INVALID), (dict(scale=-0.1), K.KV_ERR_INVALID),
])
def test_prefill_refuses(L, kw, code):
    assert _prefill(L, **kw) == code
    assert K.last_error().startswith("kvattn_prefill_chunk_fp8")


@pytest.mark.parametrize("scale", [3e38, 2.4e38])
def test_scales_past_log2(L, scale):
    """The kernels work in powers of two, with scale * log2(e): infinite, it would make NaN of
    every score of zero."""
    for call, name in ((_decode, "kvattn_decode_fp8"), (_prefill, "kvattn_prefill_chunk_fp8")):
        assert call(L, scale=scale) == K.KV_ERR_INVALID
        assert K.last_error().startswith(name) and "scale" in K.last_error()
    assert _decode(L, scale=-scale) == K.KV_ERR_INVALID


def _append(L, **kw):
    a = dict(k=A, v=A, sm=A, kv=A, nb=100, T=64, hkv=8, d=128, bs=16, dt=K.KV_BF16)
    a.update(kw)
    return L.kvattn_kv_append_fp8(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dt=5), K.KV_ERR_INVALID), (dict(T=-1), K.KV_ERR_INVALID),
    (dict(d=256), K.KV_ERR_UNSUPPORTED), (dict(d=0), K.KV_ERR_INVALID),
    (dict(hkv=0), K.KV_ERR_INVALID), (dict(hkv=1 << 16), K.KV_ERR_UNSUPPORTED),
    (dict(bs=8), K.KV_ERR_UNSUPPORTED), (dict(nb=0), K.KV_ERR_INVALID),
    (dict(nb=1 << 28), K.KV_ERR_INVALID), (dict(sm=0), K.KV_ERR_INVALID),
    (dict(v=A + 4), K.KV_ERR_INVALID),
])
def test_append_refuses(L, kw, code):
    assert _append(L, **kw) == code
    assert K.last_error().startswith("kvattn_kv_append_fp8")


def test_nothing_to_do_is_ok(L):
    assert _append(L, T=0, k=0, v=0, sm=0) == K.KV_OK
    assert _decode(L, B=0, q=0, out=0) == K.KV_OK
    assert _prefill(L, T=0, q=0, out=0) == K.KV_OK


def _map(L, **kw):
    M = 1 << 16
    a = dict(cached=A, new=A + M, S=4, free=A + 2 * M, nf=8, bt=A + 3 * M, mb=10, bs=16, T=64,
             lens=A + 4 * M, cu=A + 5 * M, slots=A + 6 * M, pos=A + 7 * M, used=A + 8 * M)
    a.update(kw)
    return L.kvattn_step_map(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(S=-1), K.KV_ERR_INVALID), (dict(nf=-1), K.KV_ERR_INVALID),
    (dict(T=-1), K.KV_ERR_INVALID), (dict(S=65536), K.KV_ERR_UNSUPPORTED),
    (dict(bs=32), K.KV_ERR_UNSUPPORTED), (dict(mb=0), K.KV_ERR_INVALID),
    (dict(mb=1 << 27), K.KV_ERR_INVALID), (dict(cached=0), K.KV_ERR_INVALID),
    (dict(free=0), K.KV_ERR_INVALID), (dict(bt=0), K.KV_ERR_INVALID),
    (dict(pos=0), K.KV_ERR_INVALID), (dict(used=0), K.KV_ERR_INVALID),
    (dict(slots=A + 6 * (1 << 16) + 2), K.KV_ERR_INVALID),
    (dict(lens=A), K.KV_ERR_INVALID),                       # in place
    (dict(lens=A + 12), K.KV_ERR_INVALID),                  # the last length
    (dict(pos=A + 6 * (1 << 16) + 252), K.KV_ERR_INVALID),  # the last slot
    (dict(used=A + 3 * (1 << 16) + 4), K.KV_ERR_INVALID),   # in the table
    (dict(cu=A + 2 * (1 << 16)), K.KV_ERR_INVALID),         # in the free list
])
def test_step_map_refuses(L, kw, code):
    assert _map(L, **kw) == code
    assert K.last_error().startswith("kvattn_step_map")


def test_binding_refuses_before_any_launch():
    q = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    bt, sl = torch.zeros(4, 3, dtype=torch.int32), torch.ones(4, dtype=torch.int32)
    kw = dict(num_kv_heads=2, max_seq_len=48)
    layer = torch.zeros(10 * K.fp8_block_bytes(2, 128), dtype=torch.uint8)
    with pytest.raises(ValueError, match="int32"):
        K.decode_fp8(q, layer, 10, bt.long(), sl, **kw)
    with pytest.raises(ValueError, match="seq_lens"):
        K.decode_fp8(q, layer, 10, bt, sl[:3], **kw)
    with pytest.raises(ValueError, match="blocks need"):
        K.decode_fp8(q, layer, 11, bt, sl, **kw)
    with pytest.raises(ValueError, match="dtype"):
        K.decode_fp8(q.half(), layer, 10, bt, sl, **kw)
    with pytest.raises(ValueError, match="out"):
        K.decode_fp8(q, layer, 10, bt, sl, out=q.float(), **kw)
    with pytest.raises(ValueError, match="contiguous"):
        K.decode_fp8(q.transpose(0, 1).contiguous().transpose(0, 1), layer, 10, bt, sl, **kw)
    with pytest.raises(ValueError, match="GPU"):
        K.decode_fp8(q, layer, 10, bt, sl, **kw)
    cu = torch.tensor([0, 2, 4], dtype=torch.int32)
    with pytest.raises(ValueError, match="cu_seqlens_q"):
        K.prefill_chunk_fp8(q, layer, 10, bt[:2], sl[:2], cu[:2], **kw)
    with pytest.raises(ValueError, match="blocks need"):
        K.prefill_chunk_fp8(q, layer[:-1], 10, bt[:2], sl[:2], cu, **kw)
    with pytest.raises(ValueError, match="GPU"):
        K.prefill_chunk_fp8(q, layer, 10, bt[:2], sl[:2], cu, **kw)
    k = torch.zeros(4, 2, 128)
    with pytest.raises(ValueError, match="shape and dtype"):
        K.kv_append_fp8(k, k.bfloat16(), sl, layer, 10)
    with pytest.raises(ValueError, match="slot_mapping"):
        K.kv_append_fp8(k, k, sl[:3], layer, 10)
    with pytest.raises(ValueError, match="blocks need"):
        K.kv_append_fp8(k, k, sl, layer, 12)
    with pytest.raises(ValueError, match="GPU"):
        K.kv_append_fp8(k, k, sl, layer, 10)


def test_binding_refuses_step_maps_before_any_launch():
    z = lambda *n: torch.zeros(*n, dtype=torch.int32)   # noqa: E731
    out = K.StepMap.empty(4, 10, "cpu")
    with pytest.raises(ValueError, match="int32"):
        K.step_map(z(4).long(), z(4), z(5), z(4, 3), max_tokens=10)
    with pytest.raises(ValueError, match="new_lens"):
        K.step_map(z(4), z(3), z(5), z(4, 3), max_tokens=10)
    with pytest.raises(ValueError, match="rows"):
        K.step_map(z(4), z(4), z(5), z(3, 3), max_tokens=10)
    with pytest.raises(ValueError, match="out"):
        K.step_map(z(4), z(4), z(5), z(4, 3), max_tokens=11, out=out)
    with pytest.raises(ValueError, match="contiguous"):
        K.step_map(z(4), z(4), z(5), z(4, 6)[:, ::2], max_tokens=10)
    with pytest.raises(ValueError, match="GPU"):
        K.step_map(z(4), z(4), z(5), z(4, 3), max_tokens=10, out=out)
