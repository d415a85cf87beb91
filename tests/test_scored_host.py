"""What the scored attention calls and the qkv appends refuse, before anything is launched:
the C ABI's checks with addresses that are never touched, the binding's with CPU tensors;
and where the tensors that they make come from when they are given a stream."""
import ctypes

import pytest
import torch

import paper_2608_23658_amd.kvattn as K
from tests.test_stream_host import HERE, KW, OTHER, _batch, _i32, notes  # noqa: F401

A = 1 << 20
M = 1 << 30
BAD, NOT_BUILT = K.KV_ERR_INVALID, K.KV_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def L():
    return K.lib()


def _scoring(a):
    cap, slopes, window = a.pop("cap"), a.pop("slopes"), a.pop("window")
    return K.Scoring(cap, slopes, window)


def _decode(L, fp8, **kw):
    a = dict(q=A, kv=A, nb=100, bt=A, sl=A, out=A, B=4, hq=32, hkv=8, d=128, bs=16, mb=10,
             msl=160, scale=0.1, s=None, dt=K.KV_BF16, ws=A, wsb=1 << 30, cap=30.0, slopes=A,
             window=64)
    a.update(kw)
    s = _scoring(a)
    a["s"] = None if kw.get("s", 0) is None else s
    return (L.kvattn_decode_scored_fp8 if fp8 else L.kvattn_decode_scored)(*a.values(), None)


def _prefill(L, fp8, **kw):
    a = dict(q=A, kv=A, nb=100, bt=A, sl=A, cu=A, out=A, B=2, T=100, budget=128, hq=32, hkv=8,
             d=128, bs=16, mb=10, msl=160, scale=0.1, s=None, dt=K.KV_BF16, ws=A, wsb=1 << 20,
             cap=30.0, slopes=A, window=64)
    a.update(kw)
    s = _scoring(a)
    a["s"] = None if kw.get("s", 0) is None else s
    call = L.kvattn_prefill_chunk_scored_fp8 if fp8 else L.kvattn_prefill_chunk_scored
    return call(*a.values(), None)


SCORES = [
    (dict(s=None), BAD), (dict(cap=-1.0), BAD), (dict(cap=float("nan")), BAD),
    (dict(cap=float("inf")), BAD), (dict(cap=2e38), BAD),   # a cap past log2(e)
    (dict(cap=1e-38, scale=10.0), BAD),                     # scale / cap
    (dict(window=-1), BAD), (dict(slopes=A + 2), BAD),
    (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD), (dict(scale=3e38), BAD),
]
COMMON = [
    (dict(bs=32), NOT_BUILT), (dict(dt=7), BAD), (dict(msl=161), BAD), (dict(nb=0), BAD),
    (dict(q=A + 8), BAD), (dict(kv=A + 8), BAD), (dict(out=0), BAD), (dict(wsb=16), BAD),
    (dict(B=-1), BAD), (dict(hq=30), BAD), (dict(d=96), NOT_BUILT), (dict(hq=24), NOT_BUILT),
]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("kw,code", SCORES + COMMON)
def test_decode_refuses(L, fp8, kw, code):
    assert _decode(L, fp8, **kw) == code
    assert K.last_error().startswith("kvattn_decode_scored" + ("_fp8" if fp8 else "") + ":")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("kw,code", SCORES + COMMON + [
    (dict(dt=K.KV_F32), NOT_BUILT), (dict(d=64), NOT_BUILT), (dict(T=200), BAD), (dict(cu=0), BAD)])
def test_prefill_refuses(L, fp8, kw, code):
    assert _prefill(L, fp8, **kw) == code
    assert K.last_error().startswith("kvattn_prefill_chunk_scored" + ("_fp8" if fp8 else "") + ":")


def test_decode_types_that_are_not_built(L):
    assert _decode(L, False, dt=K.KV_F32) == NOT_BUILT          # fp32 of 128
    assert _decode(L, True, dt=K.KV_F32, d=64) == NOT_BUILT


def test_a_windows_workspace(L):
    """At least one split's partials for every row, and no less where the window is as
    long as the context or longer."""
    big = dict(mb=1000, msl=16000, nb=1000)
    rows = 4 * 32
    one = rows * 128 * 4 + rows * 2 * 4
    assert _decode(L, False, **big, wsb=one - 1) == BAD
    for window in (0, 16000, (1 << 31) - 1):
        assert _decode(L, False, **big, wsb=2 * one, window=window) == BAD
    assert K.decode_workspace_bytes(4, 32, 128, 64 + 15) < \
        K.decode_workspace_bytes(4, 32, 128, 16000)


@pytest.mark.parametrize("fp8", [False, True])
def test_nothing_to_do_is_ok(L, fp8):
    assert _decode(L, fp8, B=0, q=0, out=0) == K.KV_OK
    assert _prefill(L, fp8, T=0, q=0, out=0) == K.KV_OK
    assert _qkv(L, fp8, T=0, q=0, k=0, v=0, sm=0, out=0, pos=0) == K.KV_OK
    assert K.last_error() == ""


def _qkv(L, fp8, **kw):
    a = dict(q=A, qs=4096, k=A + M, ks=1024, v=A + 2 * M, vs=1024, prep=None, sm=A + 3 * M,
             out=A + 4 * M, kv=A + 5 * M, nb=100, T=64, hq=32, hkv=8, d=128, bs=16, dt=K.KV_BF16)
    p = dict(qw=A + 6 * M, kw=A + 6 * M, eps=1e-6, table=A + 7 * M, n=4096, rot=128, even=0,
             pos=A + 8 * M, axes=1, sections=(64,))
    for name, value in kw.items():
        (p if name in p else a)[name] = value
    p["sections"] = (ctypes.c_int * 4)(*p["sections"])
    if kw.get("prep", 0) is not None:
        a["prep"] = K.NormRope(*p.values())
    return (L.kvattn_qkv_append_fp8 if fp8 else L.kvattn_qkv_append)(*a.values(), None)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(prep=None), BAD), (dict(dt=5), BAD), (dict(T=-1), BAD), (dict(hq=0), BAD),
    (dict(hkv=0), BAD), (dict(hkv=1 << 15), NOT_BUILT), (dict(hq=65535), NOT_BUILT),
    (dict(d=0), BAD), (dict(d=256), NOT_BUILT), (dict(bs=8), NOT_BUILT), (dict(nb=0), BAD),
    (dict(nb=1 << 27), BAD), (dict(eps=-1e-6), BAD), (dict(eps=float("nan")), BAD),
    (dict(qw=A + 8), BAD), (dict(kw=A + 2), BAD), (dict(table=A + 7 * M + 8), BAD),
    (dict(n=0), BAD), (dict(rot=0), BAD), (dict(rot=33), BAD), (dict(rot=256), BAD),
    (dict(d=64, rot=128), BAD), (dict(rot=96, sections=(48,)), NOT_BUILT), (dict(axes=0), BAD),
    (dict(axes=5), BAD), (dict(sections=(63,)), BAD),
    (dict(axes=2, sections=(-1, 65)), BAD), (dict(axes=3, sections=(64, 64, 64)), BAD),
    (dict(axes=2, sections=((1 << 31) - 1, (1 << 31) - 1)), BAD),
    (dict(pos=0), BAD), (dict(pos=A + 2), BAD), (dict(q=0), BAD), (dict(v=0), BAD),
    (dict(sm=0), BAD), (dict(out=0), BAD), (dict(kv=0), BAD), (dict(k=A + M + 8), BAD),
    (dict(kv=A + 5 * M + 4), BAD), (dict(qs=4100), BAD), (dict(vs=(1 << 40) + 8), BAD),
    # what is written over something else: the layer, a token's rows, the last of a table
    (dict(out=A + 5 * M), BAD), (dict(out=A + M), BAD), (dict(out=A, qs=6144), BAD),
    (dict(out=A + 16), BAD), (dict(kv=A + 7 * M + 4096 * 512 - 16), BAD),
    (dict(kv=A + 2 * M + 63 * 2048 + 2032), BAD), (dict(out=A + 8 * M), BAD),
])
def test_qkv_append_refuses(L, fp8, kw, code):
    assert _qkv(L, fp8, **kw) == code
    assert K.last_error().startswith("kvattn_qkv_append" + ("_fp8" if fp8 else "") + ":")


# ---- the binding ----
T, HQ, HKV, D = 6, 8, 2, 128


def _rows(dtype=torch.bfloat16):
    return [torch.zeros(T, h, D, dtype=dtype) for h in (HQ, HKV, HKV)]


def _layer(fp8, blocks=10):
    return torch.zeros(blocks * (K.fp8_block_bytes(HKV, D) if fp8 else 2 * HKV * 16 * D * 2),
                       dtype=torch.uint8)


@pytest.mark.parametrize("fp8", [False, True])
def test_binding_refuses_rows(fp8):
    call = K.qkv_append_fp8 if fp8 else K.qkv_append
    q, k, v = _rows()
    slots, table, pos = _i32(T), torch.zeros(32, D), _i32(T)
    w = torch.zeros(D, dtype=torch.bfloat16)

    def refused(match, q=q, k=k, v=v, slots=slots, blocks=10, **kw):
        with pytest.raises(ValueError, match=match):
            call(q, k, v, slots, _layer(fp8), blocks, **kw)

    refused("one dtype", k=k[:5])
    refused("one dtype", v=v.float())
    refused("one dtype", v=torch.zeros(T, 4, D, dtype=torch.bfloat16))
    refused("contiguous", q=torch.zeros(T, D, HQ, dtype=torch.bfloat16).transpose(1, 2))
    refused("contiguous", k=torch.zeros(T, 4, D, dtype=torch.bfloat16)[:, ::2])
    refused("slot_mapping", slots=slots.long())
    refused("slot_mapping", slots=slots[:5])
    refused("blocks need", blocks=11)
    refused("q_weight", q_weight=w.float())
    refused("k_weight", k_weight=w[:64])
    refused("rope_table must", rope_table=table.double(), positions=pos)
    refused("positions must", rope_table=table)
    refused("positions must", rope_table=table, positions=pos.long())
    refused("positions must", rope_table=table, positions=pos[:5])
    refused("need a rope_table", positions=pos)
    refused("need a rope_table", sections=(64,))
    refused("need sections", rope_table=table, positions=_i32(2, T))
    refused("sections", rope_table=table, positions=_i32(2, T), sections=(64,))
    refused("sections", rope_table=table, positions=_i32(5, T), sections=(64, 0, 0, 0, 0))
    refused("out must", out=q[:5])
    refused("out must", out=q.float())
    with pytest.raises(ValueError, match="CUDA|cuda|GPU"):
        call(q, k, v, slots, _layer(fp8), 10)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("chunk", [False, True])
def test_binding_refuses_scores(fp8, chunk):
    call = getattr(K, ("prefill_chunk" if chunk else "decode") + "_scored" + ("_fp8" if fp8 else ""))
    q = _rows()[0]
    table, lens, cu = _i32(T, 3), _i32(T), _i32(T + 1)

    def refused(match, q=q, table=table, lens=lens, blocks=10, **kw):
        args = (q, _layer(fp8), blocks, table, lens) + ((cu,) if chunk else ())
        with pytest.raises(ValueError, match=match):
            call(*args, num_kv_heads=HKV, max_seq_len=48, **kw)

    refused("slopes", slopes=torch.zeros(HQ + 1))
    refused("slopes", slopes=torch.zeros(HQ, dtype=torch.bfloat16))
    refused("slopes", slopes=torch.zeros(1, HQ))
    refused("int32", table=table.long())
    refused("must have 3 rows" if chunk else "seq_lens", lens=lens[:3])
    refused("blocks need", blocks=11)
    refused("out", out=q[:3])
    refused("CUDA|cuda|GPU")


SCORED = dict(softcap=30.0, slopes=torch.zeros(8), window=20)


def _qkv_args():
    q, k, v = _rows()
    return q, k, v, _i32(T), torch.zeros(1 << 17, dtype=torch.uint8), 2


CALLS = {
    "decode_scored": lambda **kw: K.decode_scored(*_batch(), **KW, **SCORED, **kw),
    "decode_scored_fp8": lambda **kw: K.decode_scored_fp8(*_batch(), **KW, **SCORED, **kw),
    "prefill_chunk_scored": lambda **kw: K.prefill_chunk_scored(*_batch(), _i32(5), **KW,
                                                                **SCORED, **kw),
    "prefill_chunk_scored_fp8": lambda **kw: K.prefill_chunk_scored_fp8(
        *_batch(), _i32(5), **KW, **SCORED, **kw),
    "qkv_append": lambda **kw: K.qkv_append(*_qkv_args(), **kw),
    "qkv_append_fp8": lambda **kw: K.qkv_append_fp8(*_qkv_args(), **kw),
}


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("stream,handle", [(OTHER, 0x2000), (0x3000, 0x3000), (0, 0)])
def test_made_for_the_stream_of_the_call(notes, name, stream, handle):  # noqa: F811
    got = CALLS[name](stream=stream)
    made = [on for _, on in notes.made]
    assert made and all(on == handle for on in made), "made for another stream"
    assert (got.data_ptr(), HERE.cuda_stream) in notes.recorded
    assert notes.on is HERE


@pytest.mark.parametrize("name", sorted(CALLS))
def test_made_for_the_current_stream_without_one(notes, name):  # noqa: F811
    CALLS[name]()
    assert notes.made and all(on == HERE.cuda_stream for _, on in notes.made)
    assert not notes.recorded


# ---- what the binding hands to the library ----
class _Asked(Exception):
    pass


def _asked(monkeypatch):
    """Calls of the library end in _Asked, with its arguments."""
    class Library:
        def __getattr__(self, name):
            def call(*a):
                if name.endswith("bytes"):
                    return 4096
                raise _Asked(*a)
            return call
    monkeypatch.setattr(K, "lib", Library)
    monkeypatch.setattr(K, "_require_here", lambda *ts: None)
    monkeypatch.setattr(K, "_stream", lambda stream: 0)


WIDE = [(1 << 32) + 5, 1 << 31, -(1 << 31) - 1, 1 << 64]


@pytest.mark.parametrize("wide", WIDE)
@pytest.mark.parametrize("name", sorted(n for n in CALLS if "scored" in n))
def test_integers_past_32_bits_are_refused(monkeypatch, name, wide):
    """ctypes would cut a window of 2^32 + 5 to one of 5."""
    _asked(monkeypatch)
    monkeypatch.setitem(SCORED, "window", wide)
    with pytest.raises(ValueError, match="window .* 32 bits"):
        CALLS[name]()
    monkeypatch.setitem(SCORED, "window", 20)
    monkeypatch.setitem(KW, "max_seq_len", wide)
    with pytest.raises(ValueError, match="max_seq_len .* 32 bits"):
        CALLS[name]()


@pytest.mark.parametrize("name", sorted(n for n in CALLS if "scored" in n))
def test_what_the_library_refuses_reaches_it(monkeypatch, name):
    _asked(monkeypatch)
    monkeypatch.setitem(SCORED, "window", -1)
    with pytest.raises(_Asked) as e:
        CALLS[name]()
    scoring = next(x for x in e.value.args if isinstance(x, K.Scoring))
    assert (scoring.softcap, scoring.window) == (30.0, -1)


@pytest.mark.parametrize("name", sorted(n for n in CALLS if "scored" in n))
def test_a_cap_that_fp32_rounds_to_zero_is_refused(monkeypatch, name):
    _asked(monkeypatch)
    monkeypatch.setitem(SCORED, "softcap", 1e-60)
    with pytest.raises(ValueError, match="softcap"):
        CALLS[name]()


@pytest.mark.parametrize("name", ["qkv_append", "qkv_append_fp8"])
def test_sections_and_blocks_past_32_bits_are_refused(monkeypatch, name):
    _asked(monkeypatch)
    q, k, v, slots, layer, _ = _qkv_args()
    rope = dict(rope_table=torch.zeros(32, D), positions=_i32(2, T))
    with pytest.raises(ValueError, match="section .* 32 bits"):
        getattr(K, name)(q, k, v, slots, 0, 2, **rope, sections=((1 << 32) + 60, 4))
    with pytest.raises(ValueError, match="num_blocks .* 32 bits"):
        getattr(K, name)(q, k, v, slots, 0, (1 << 32) + 2)


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("dtype,right", [(torch.bfloat16, "own"), (torch.float32, None),
                                         (torch.float16, None), (torch.float8_e4m3fn, "8bit"),
                                         (torch.float8_e5m2, None), (torch.uint8, "both"),
                                         (torch.int16, "both")])
def test_a_layer_of_another_type_is_refused(monkeypatch, name, dtype, right):
    """Rows in bf16 over a layer tensor in fp32, say, whose bytes would do."""
    _asked(monkeypatch)
    layer = torch.zeros(1 << 18, dtype=dtype)
    if "qkv" in name:
        args = _qkv_args()[:4] + (layer, 2)
        kw = {}
    else:
        q, _, blocks, *rest = _batch()
        args = (q, layer, blocks, *rest) + ((_i32(5),) if "prefill" in name else ())
        kw = {**KW, **SCORED}
    ok = right in ("both", "8bit" if name.endswith("fp8") else "own")
    with pytest.raises(_Asked if ok else ValueError, match=None if ok else "kv_layer is"):
        getattr(K, name)(*args, **kw)


@pytest.mark.parametrize("name", ["qkv_append", "qkv_append_fp8"])
def test_one_tokens_stride_does_not_count(monkeypatch, name):
    """torch gives a dimension of one any stride: a row that was a column's, say."""
    _asked(monkeypatch)
    q, k, v = (torch.zeros(h, D, 1, dtype=torch.bfloat16).permute(2, 0, 1) for h in (HQ, HKV, HKV))
    assert q.is_contiguous() and q.stride(0) == 1
    with pytest.raises(_Asked) as e:
        getattr(K, name)(q, k, v, _i32(1), torch.zeros(1 << 17, dtype=torch.uint8), 2)
    assert [e.value.args[i] for i in (1, 3, 5)] == [HQ * D, HKV * D, HKV * D]
    q = torch.zeros(T, HQ + 4, D, dtype=torch.bfloat16)[:, :HQ]
    with pytest.raises(_Asked) as e:
        getattr(K, name)(q, *_rows()[1:], _i32(T), torch.zeros(1 << 17, dtype=torch.uint8), 2)
    assert e.value.args[1] == (HQ + 4) * D
