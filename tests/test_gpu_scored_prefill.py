"""Chunked prefill with capped, biased and windowed scores against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_23658_amd.kvattn as K
from tests.gpu_helpers import f64, require_gpu, say
from tests.scored_helpers import MODS, Call, assert_scored, assert_scored_f32
from tests.test_gpu_scored_decode import _poison

pytestmark = pytest.mark.gpu
CACHES = ["bf16", "8bit"]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _small(c):
    """The least workspace a call takes: every tile is one workgroup's."""
    T = c.b.total_q_tokens
    return K.workspace(-(-(8 * (T // 32 + c.b.num_seqs + 1) + 16) // 256) * 256)


@pytest.mark.parametrize("hq,hkv", [(32, 8), (4, 4), (16, 8), (16, 2), (12, 3)])
@pytest.mark.parametrize("mods", sorted(MODS))
@pytest.mark.parametrize("cache", CACHES)
def test_ragged(hq, hkv, mods, cache):
    """Chunks from one row on, over contexts of any length, and one-row sequences."""
    say("prefill scored", cache, hq, hkv, mods)
    lens = [1, 16, 17, 64, 65, 130, 300, 700, 1025, 900]
    new = [1, 16, 3, 64, 1, 130, 100, 1, 257, 40]
    c = Call(lens, new, hq=hq, hkv=hkv, d=128, cache=cache, seed=hq, **MODS[mods])
    c.check(c.prefill(), False, f"{cache} {hq}/{hkv} {mods}")


@pytest.mark.parametrize("lens,new,hq,hkv,window", [
    ([1], [1], 8, 1, 1), ([33], [33], 8, 1, 0), ([128], [64], 8, 2, 0), ([200], [7], 32, 8, 50),
    ([3000], [1], 16, 2, 0), ([3000], [1], 16, 2, 2900),     # one row alone
    ([6150], [201], 8, 2, 0), ([6150], [201], 8, 2, 4000),   # tiles shared by several workgroups
    ([2500, 1700, 1200], [1, 1, 300], 8, 1, 0), ([2500, 1700, 1200], [1, 1, 300], 8, 1, 1400),
    ([40] * 30, [40] * 30, 8, 8, 9), ([64, 64], [0, 64], 8, 2, 33),
    ([300] * 5 + [1100] * 3, [1] * 5 + [2] * 3, 32, 8, 500),
])
@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("small", [False, True])
@pytest.mark.parametrize("softcap", [0.0, 15.0])
def test_by_plan(lens, new, hq, hkv, window, cache, small, softcap):
    say("prefill scored", lens[:4], new[:4], hq, hkv, window, cache, softcap)
    c = Call(lens, new, hq=hq, hkv=hkv, d=128, cache=cache, seed=sum(lens), window=window,
             softcap=softcap, bias=not window and not softcap)
    out = c.prefill(ws=_small(c) if small else None)
    c.check(out, False, f"{cache} {len(lens)} {sum(new)} window {window} cap {softcap}")


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 500, 1000,
                                    2 ** 31 - 1])
def test_windows(cache, window):
    """Windows narrower than a tile's rows, of whole steps and not, and past all keys."""
    say("prefill window", cache, window)
    c = Call([700, 333, 1500], [300, 333, 65], hq=8, hkv=2, d=128, cache=cache,
             seed=window % 1000, window=window)
    c.check(c.prefill(), False, f"{cache} window {window}")
    c.check(c.prefill(ws=_small(c)), False, f"{cache} window {window}, whole tiles")


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("window", [20, 100, 1000])
@pytest.mark.parametrize("softcap", [0.0, 20.0])
def test_what_lies_before_a_window(cache, window, softcap):
    """As for decode: entries of blocks before the first row's window are -1, beyond the layer
    or another's, and what that window's first block holds before it is NaN."""
    say("prefill poisoned", cache, window)
    lens, new = [window + 31, 1700, 2048, 1111, 1500], [30, 1, 200, 64, 1]
    c = Call(lens, new, hq=8, hkv=2, d=128, cache=cache, window=window, softcap=softcap)
    small = _small(c)
    want, whole = c.prefill(), c.prefill(ws=small)
    c.check(want, False, f"{cache} window {window}")
    c.check(whole, False, f"{cache} window {window}, whole tiles")
    dead = torch.zeros(c.b.num_blocks, 16, dtype=torch.bool)
    for s, (L, n) in enumerate(zip(lens, new)):
        first = max(0, L - n - window + 1)
        row = c.b.block_table[s]
        dead[row[first // 16], :first % 16] = True
        row[:first // 16] = ([-1, 10 ** 9, c.b.num_blocks, 0] * 64)[:first // 16]
    c.kv = c.kv.clone()
    _poison(c.kv, dead, c)
    c.set_table()
    assert torch.equal(want.view(torch.int16), c.prefill().view(torch.int16))
    assert torch.equal(whole.view(torch.int16), c.prefill(ws=small).view(torch.int16))


@pytest.mark.parametrize("cache", CACHES)
def test_with_nothing_it_is_prefill(cache):
    say("prefill scored plain", cache)
    c = Call([1, 70, 900, 2100, 333], [1, 70, 33, 1, 300], hq=8, hkv=2, d=128, cache=cache)
    plain = K.prefill_chunk_fp8 if cache == "8bit" else K.prefill_chunk
    want = plain(c.q, c.kv, c.b.num_blocks, c.bt, c.sl, c.cu, num_kv_heads=2,
                 max_seq_len=c.b.max_seq_len, scale=c.scale)
    assert torch.equal(want.view(torch.int16), c.prefill().view(torch.int16))


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("softcap,q_size", [(1.0, 50.0), (50.0, 40.0), (0.01, 1.0), (3e37, 4.0)])
def test_caps(cache, softcap, q_size):
    say("prefill caps", cache, softcap)
    c = Call([90, 700, 20], [33, 200, 1], hq=4, hkv=2, d=128, cache=cache, softcap=softcap,
             q_size=q_size)
    c.mods["softcap"] = min(softcap, 1e6)      # a cap no score feels, for the bound
    ref, weight = c.expected(False)
    c.mods["softcap"] = softcap
    from tests.scored_helpers import assert_scored
    assert_scored(c.prefill(), ref, weight, cache, min(softcap, 200.0), f"{cache} cap {softcap}")


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("mods", [dict(softcap=10.0), dict(window=50), dict(bias=True)])
def test_a_negative_scale_and_zero(cache, mods):
    for scale in (-0.2, 0.0):
        c = Call([5, 300, 700], [5, 100, 1], hq=4, hkv=2, d=128, cache=cache, scale=scale,
                 q_size=1.0, **mods)
        c.check(c.prefill(), False, f"{cache} scale {scale} {mods}")


@pytest.mark.parametrize("cache", CACHES)
def test_ids_outside_empty_rows_and_padding(cache):
    """Ids outside the layer contribute nothing, a row that sees no key gets zeros, and rows
    behind the last sequence's stay."""
    say("prefill scored ids", cache)
    c = Call([200, 90, 130], [50, 20, 1], hq=4, hkv=2, d=128, cache=cache, window=40, softcap=9.0)
    c.b.block_table[0, 7] = c.b.num_blocks + 3
    c.b.block_table[0, 11] = -2
    c.b.block_table[1, :] = -1
    c.set_table()
    pad = torch.full((9, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    c.q = torch.cat([c.q, pad])
    out = torch.full_like(c.q, 5.0)
    c.prefill(out=out)
    c.check(out[:71], False, f"{cache} ids outside")
    assert not out[50:70].any() and (out[71:] == 5.0).all()


def test_chunks_of_a_prompt_are_the_prompt():
    """A prompt in chunks gives what it gives at once, bit for bit where tiles are whole."""
    for cache in CACHES:
        c = Call([600], [600], hq=8, hkv=2, d=128, cache=cache, window=150, softcap=20.0)
        small = _small(c)
        whole = c.prefill(ws=small)
        q, parts = c.q, []
        for a in range(0, 600, 128):
            b = min(600, a + 128)
            c.q = q[a:b].contiguous()
            c.sl = torch.tensor([b], dtype=torch.int32, device="cuda")
            c.cu = torch.tensor([0, b - a], dtype=torch.int32, device="cuda")
            parts.append(c.prefill(ws=small, max_seq_len=b))
        parts = torch.cat(parts)
        ref, weight = None, None
        c.b.q = q.cpu()
        ref, weight = c.expected(False)
        from tests.scored_helpers import assert_scored
        assert_scored(parts, ref, weight, cache, 20.0, f"{cache} chunks")
        assert torch.allclose(parts.float(), whole.float(), atol=2e-2)


def test_streams_and_graphs():
    """As for decode, over a step of a chunk and one-row sequences."""
    lens, new = [1500, 40, 900, 2048], [300, 1, 1, 64]
    c = Call(lens, new, hq=8, hkv=2, d=128, softcap=20.0, window=700, bias=True)
    want = c.prefill()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.prefill(stream=side)
    torch.cuda.synchronize()
    assert torch.equal(want, got)
    T = sum(new)
    kw = dict(out=torch.empty_like(c.q), ws=K.workspace(K.prefill_workspace_bytes(4, T, 8, 128)),
              max_seq_len=2048)
    c.prefill(**kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.prefill(**kw)
    for turn in range(4):
        c.sl.copy_(torch.tensor([n - 37 * turn if n > 500 else n for n in lens]))
        want = c.prefill(max_seq_len=2048)
        kw["out"].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, kw["out"]), turn


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("mods", [dict(), dict(softcap=20.0), dict(bias=True)])
@pytest.mark.parametrize("window", [20, 90, 1000])
def test_ids_behind_a_window_may_be_others(cache, mods, window):
    """Entries of blocks before the first row's window still name blocks of the layer, which
    others have by now and which hold anything: NaN here, in every slot and exponent."""
    say("prefill stale ids", cache, mods, window)
    lens, new = [window + 31, 1700, 2048, 1111, 1500], [30, 1, 200, 64, 1]
    c = Call(lens, new, hq=8, hkv=2, d=128, cache=cache, window=window, **mods)
    small = _small(c)
    want, whole = c.prefill(), c.prefill(ws=small)
    c.check(want, False, f"{cache} window {window} {mods}")
    c.check(whole, False, f"{cache} window {window} {mods}, whole tiles")
    given_up = []
    for s, (L, n) in enumerate(zip(lens, new)):
        given_up += list(c.b.block_table[s][:max(0, L - n - window + 1) // 16])
    layer = c.kv.clone().view(c.b.num_blocks, -1)
    layer[torch.tensor(sorted(given_up)).cuda()] = 0xff if cache == "8bit" else float("nan")
    c.kv = layer.view(c.kv.shape)
    assert torch.equal(want.view(torch.int16), c.prefill().view(torch.int16))
    assert torch.equal(whole.view(torch.int16), c.prefill(ws=small).view(torch.int16))


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("softcap", [1e4, 1e5, 1e6])
def test_a_large_product_beside_small_ones_under_a_large_cap(cache, softcap):
    """One row's products pass half the cap, the others' scores are of a few units: theirs are
    as exact as under a small cap (off by at most 2^-19 of themselves)."""
    say("prefill large cap", cache, softcap)
    for lens, new, big in (([40], [33], 5), ([700, 90], [200, 40], 150)):
        c = Call(lens, new, hq=4, hkv=2, d=128, cache=cache, softcap=softcap, seed=11)
        # every head of one row: a query along a key that it sees, of 0.8 caps
        k, _ = oracle.gather_kv(c.b.kv_raw(), c.b.dtype, c.b.block_table[0], lens[0], 2, 16, 128)
        at = lens[0] - new[0] + big
        for h in range(4):
            key = torch.from_numpy(k[at - 3, h // 2]).float()
            row = key * (0.8 * softcap / (float(key @ key) * c.scale))
            c.b.q[big, h] = row.to(c.b.q.dtype)
        c.q = c.b.q.cuda()
        got = f64(c.prefill())
        ref, weight = c.expected(False)
        others = np.arange(sum(new)) != big
        what = f"{cache} cap {softcap} of {lens}"
        assert_scored(got[others], ref[others], weight[others], cache, 0.0, what)
        # its own: 2^-19 of scores up to the cap; the key it points at is most of the sum
        assert_scored(got[big], ref[big], weight[big], cache, 4 * softcap, what + ", its row")


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("decode", [False, True])
def test_a_cap_at_a_tiny_scale(cache, decode):
    """Queries of 2^40 at a scale of 2^-40: the scores of a plain call, half a cap large, whose
    quotient of scale and cap leaves a polynomial's coefficients no place in fp32."""
    say("tiny scale", cache, decode)
    c = Call([20, 33], [1, 1] if decode else [20, 30], hq=4, hkv=2, d=128, cache=cache,
             softcap=30.0, scale=128 ** -0.5 * 2.0 ** -40)
    c.b.q = (c.b.q.float() * 2.0 ** 40).to(c.b.q.dtype)
    c.q = c.b.q.cuda()
    c.check(c.decode() if decode else c.prefill(), decode, f"{cache} tiny scale, decode {decode}")


@pytest.mark.parametrize("cache,d", [("bf16", 128), ("f32", 64), ("8bit", 64)])
def test_a_cap_past_every_score_leaves_them(cache, d):
    """scale / softcap below fp32's least value: the scores are those of no cap."""
    say("decode, a cap of 1e38", cache)
    c = Call([5, 300], [1, 1], hq=4, hkv=2, d=d, cache=cache, scale=1e-8, q_size=1e8)
    (ref, weight), kw = c.expected(True), dict(softcap=1e38)
    if cache == "f32":
        assert_scored_f32(c.decode(**kw), ref, weight, 300, c.score_size(), "f32 decode")
    else:
        assert_scored(c.decode(**kw), ref, weight, cache, 0.0, f"{cache} decode")
    if d == 128:
        c = Call([60, 300], [30, 9], hq=4, hkv=2, d=d, cache=cache, scale=1e-8, q_size=1e8)
        assert_scored(c.prefill(**kw), *c.expected(False), cache, 0.0, f"{cache} prefill")


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("shift", [10, 15, 20, 30, 60, 100])
@pytest.mark.parametrize("q_size", [4.0, 1.0, 0.25, 2.0 ** -9])
def test_caps_at_scales_that_leave_a_polynomial_fewer_terms(cache, shift, q_size):
    """Queries of 2^shift at a scale of 2^-shift: the coefficients of a step of small products
    leave fp32 one after another, and with them the products that are taken as small, down from
    half the cap; at the last shifts the products' squares leave it too."""
    say("prefill scales", cache, shift, q_size)
    c = Call([20, 33, 300], [20, 30, 70], hq=4, hkv=2, d=128, cache=cache, softcap=30.0,
             q_size=q_size, scale=128 ** -0.5 * 2.0 ** -shift)
    c.b.q = (c.b.q.float() * 2.0 ** shift).to(c.b.q.dtype)
    c.q = c.b.q.cuda()
    c.check(c.prefill(), False, f"{cache} 2^-{shift} {q_size}")
