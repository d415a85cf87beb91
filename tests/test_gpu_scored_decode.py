"""Decode with capped, biased and windowed scores against the fp64 oracle."""
import numpy as np
import pytest
import torch

import paper_2608_23658_amd.kvattn as K
from tests.gpu_helpers import require_gpu, say
from tests.scored_helpers import MODS, Call, assert_scored, assert_scored_f32

pytestmark = pytest.mark.gpu
RAGGED = [1, 15, 16, 17, 63, 64, 65, 99, 100, 101, 115, 116, 511, 1024, 1025, 1500, 2049, 4097]
HEADS = [("bf16", 32, 8, 128), ("bf16", 2, 2, 128), ("bf16", 16, 8, 128), ("bf16", 24, 3, 128),
         ("bf16", 16, 2, 64), ("bf16", 3, 3, 64), ("f32", 8, 1, 64), ("f32", 4, 2, 64),
         ("f32", 8, 2, 64), ("f32", 3, 3, 64), ("8bit", 32, 8, 128), ("8bit", 24, 3, 128),
         ("8bit", 16, 2, 64), ("8bit", 2, 2, 128)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("cache,hq,hkv,d", HEADS)
@pytest.mark.parametrize("mods", sorted(MODS))
def test_ragged(cache, hq, hkv, d, mods):
    say("decode scored", cache, hq, hkv, d, mods)
    c = Call(RAGGED, [1] * len(RAGGED), hq=hq, hkv=hkv, d=d, cache=cache, seed=hq + d,
             **MODS[mods])
    c.check(c.decode(), True, f"{cache} {hq}/{hkv}/{d} {mods}")


@pytest.mark.parametrize("cache,d", [("bf16", 128), ("f32", 64), ("8bit", 64)])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 63, 64, 65, 1009, 1010, 1024, 1025, 3000,
                                    2 ** 31 - 1])
def test_windows(cache, d, window):
    """Windows that begin at every place of a block, end a split, or hold everything."""
    say("decode window", cache, window)
    lens = [1, 16, 17, 64, 1024, 1030, 2047, 2048, 3001]
    c = Call(lens, [1] * len(lens), hq=4, hkv=2, d=d, cache=cache, seed=window % 1000,
             window=window)
    c.check(c.decode(), True, f"{cache} window {window}")


@pytest.mark.parametrize("lens,bound,window", [
    ([3971], 3971, 0), ([3971], 3971, 3000),         # a workgroup per wavefront
    ([37], 4096, 0), ([1], 1, 1), ([5000, 1, 9000, 700], 9000, 2500),
    ([20] * 40 + [300], 131072, 0),                  # far more workgroups than work
    ([20] * 40 + [300], 131072, 200), ([200] * 300, 200, 64),
    ([700] * 200 + [9000], 131072, 5000),
])
@pytest.mark.parametrize("cache,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("8bit", 128)])
def test_by_launch(lens, bound, window, cache, d):
    say("decode scored", len(lens), bound, window, cache, d)
    c = Call(lens, [1] * len(lens), hq=8, hkv=1, d=d, cache=cache, seed=len(lens), softcap=30.0,
             window=window)
    short = bound // 16 + 1 - c.b.block_table.shape[1]
    c.b.block_table = np.pad(c.b.block_table, ((0, 0), (0, max(0, short))), constant_values=-1)
    c.set_table()
    c.check(c.decode(max_seq_len=bound), True, f"{len(lens)} under {bound}, {cache} {d}")


@pytest.mark.parametrize("cache,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("8bit", 128)])
@pytest.mark.parametrize("window", [33, 100, 1500])
def test_what_lies_before_a_window(cache, d, window):
    """Blocks before the window are given up: their entries are -1, beyond the layer or
    another's; what the window's first block holds before it is NaN, in K and in V."""
    say("decode poisoned", cache, window)
    lens = [window + 1, window + 7, 2000, 2040, 3003]
    c = Call(lens, [1] * len(lens), hq=8, hkv=2, d=d, cache=cache, window=window)
    want = c.decode()
    c.check(want, True, f"{cache} window {window}")
    layer = c.kv.clone()
    dead = torch.zeros(c.b.num_blocks, 16, dtype=torch.bool)
    for s, L in enumerate(lens):
        first = L - window
        row = c.b.block_table[s]
        dead[row[first // 16], :first % 16] = True
        row[:first // 16] = ([-1, 10 ** 9, c.b.num_blocks, 0] * 64)[:first // 16]
    _poison(layer, dead, c)
    c.kv = layer
    c.set_table()
    assert torch.equal(want.view(torch.uint8), c.decode().view(torch.uint8))


def _poison(layer, dead, c):
    """NaN in the slots ``dead`` [blocks, 16] of every head's K and V."""
    from oracle import fp8
    hkv, d, dead = c.b.num_kv_heads, c.b.head_dim, dead.cuda()
    if c.cache == "8bit":
        t = layer.view(c.b.num_blocks, -1)
        r, j = np.arange(16)[:, None], np.arange(d)[None, :]
        for kind in range(2):
            place = torch.from_numpy(fp8.place(kind, r, j)).cuda()
            for g in range(hkv):
                at = (kind * hkv + g) * 16 * d + place
                x = t[:, at]
                t[:, at] = torch.where(dead[:, :, None], torch.full_like(x, 0x7f), x)
        return
    vec = 16 // layer.element_size()
    t = layer.view(c.b.num_blocks, 2, hkv, 16 * d)
    k = t[:, 0].view(-1, hkv, d // vec, 16, vec)
    k.masked_fill_(dead[:, None, None, :, None], float("nan"))
    t[:, 1].view(-1, hkv, d, 16).masked_fill_(dead[:, None, None, :], float("nan"))


@pytest.mark.parametrize("cache,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("8bit", 128)])
def test_with_nothing_it_is_decode(cache, d):
    """No cap, no bias, no window: the plain call's bits."""
    say("decode scored plain", cache)
    c = Call([1, 70, 900, 2100, 333], [1] * 5, hq=8, hkv=2, d=d, cache=cache)
    plain = K.decode_fp8 if cache == "8bit" else K.decode
    want = plain(c.q, c.kv, c.b.num_blocks, c.bt, c.sl, num_kv_heads=2,
                 max_seq_len=c.b.max_seq_len, scale=c.scale)
    assert torch.equal(want.view(torch.uint8), c.decode().view(torch.uint8))


@pytest.mark.parametrize("cache,d", [("bf16", 128), ("f32", 64), ("8bit", 64)])
@pytest.mark.parametrize("softcap,q_size", [(1.0, 50.0), (50.0, 40.0), (0.01, 1.0), (1e4, 30.0),
                                            (3e37, 4.0)])
def test_caps(cache, d, softcap, q_size):
    """From scores that are all at the cap to a cap that no score feels."""
    say("decode caps", cache, softcap)
    lens = [1, 20, 130, 700]
    c = Call(lens, [1] * 4, hq=4, hkv=2, d=d, cache=cache, softcap=softcap, q_size=q_size)
    ref, weight = c.expected(True)
    what = f"{cache} cap {softcap}"
    if cache == "f32":
        assert_scored_f32(c.decode(), ref, weight, max(lens), c.score_size(), what)
    else:                        # a cap no score feels is off by 2^-21 of the scores, not of it
        assert_scored(c.decode(), ref, weight, cache, min(softcap, 200.0), what)


@pytest.mark.parametrize("cache,d", [("bf16", 128), ("f32", 64), ("8bit", 128)])
def test_a_negative_scale(cache, d):
    c = Call([5, 300, 1100], [1] * 3, hq=4, hkv=2, d=d, cache=cache, softcap=10.0, scale=-0.2,
             q_size=1.0)
    c.check(c.decode(), True, "negative scale")


def test_infinite_products_meet_the_cap():
    """q . k beyond fp32: the score is the cap, of its sign. (One product alone is not zero: of
    two infinite ones of other signs the sum is NaN, with a cap or without.)"""
    c = Call([40], [1], hq=2, hkv=1, d=64, cache="f32", softcap=4.0, q_size=1.0, scale=8.0)
    c.q.zero_()
    c.q[:, :, 5] = 3e38
    c.b.q.copy_(c.q.cpu())
    c.check(c.decode(), True, "infinite products")


def test_an_empty_sequence_and_ids_outside():
    for cache, d in (("bf16", 128), ("f32", 64), ("8bit", 128)):
        c = Call([200, 30, 90], [1] * 3, hq=4, hkv=2, d=d, cache=cache, window=120, softcap=9.0)
        c.b.seq_lens[1] = 0
        c.b.block_table[0, 7] = c.b.num_blocks + 3
        c.b.block_table[2, :] = -1                      # nothing is left of it
        c.set_table()
        out = c.decode()
        c.check(out, True, f"{cache} empty")
        assert not out[1].any() and not out[2].any()


def test_a_sequence_alone_and_in_a_batch():
    """A sequence's bits depend on itself."""
    lens = [700, 5000, 33, 2600] * 12
    for cache in ("bf16", "8bit"):
        c = Call(lens, [1] * len(lens), hq=8, hkv=2, d=128, cache=cache, **MODS["all"])
        whole = c.decode()
        c.q, c.bt, c.sl = c.q[5:6].clone(), c.bt[5:6].clone(), c.sl[5:6].clone()
        assert torch.equal(whole[5:6].view(torch.int16), c.decode().view(torch.int16))


def test_streams_and_graphs():
    """On a stream that is not the current one, and captured, with the lengths changing between
    replays and eager calls between them."""
    lens = [1500, 40, 900, 2048]
    c = Call(lens, [1] * 4, hq=8, hkv=2, d=128, softcap=20.0, window=700, bias=True)
    want = c.decode()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.decode(stream=side)
    torch.cuda.synchronize()
    assert torch.equal(want, got)
    kw = dict(out=torch.empty_like(c.q), ws=K.workspace(K.decode_workspace_bytes(4, 8, 128, 715)),
              max_seq_len=2048)
    c.decode(**kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.decode(**kw)
    for turn in range(4):
        c.sl.copy_(torch.tensor([n - 37 * turn if n > 200 else n for n in lens]))
        want = c.decode()
        kw["out"].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, kw["out"]), turn
