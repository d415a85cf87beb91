"""Biases that are steep, and that favour far keys, against the fp64 oracle: there a row's
largest scores come last, so that the softmax's reference moves at step after step."""
import numpy as np
import pytest
import torch

import paper_2608_23658_amd.kvattn as K
from tests.gpu_helpers import f64, require_gpu, say
from tests.scored_helpers import Call, assert_scored_f32

pytestmark = pytest.mark.gpu
SLOPES = np.array([8.0, 1.0, -0.05, -1.0, -8.0, 0.3, 0.0, -2.5], dtype=np.float32)
MODS = {"bias": dict(), "cap": dict(softcap=20.0), "window": dict(window=333),
        "both": dict(softcap=5.0, window=900)}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _call(lens, new, d, cache, **kw):
    c = Call(lens, new, hq=8, hkv=2, d=d, cache=cache, seed=sum(lens), bias=True, **kw)
    c.slopes = SLOPES
    c.dev_slopes = torch.from_numpy(SLOPES).cuda()
    return c


def _check(c, got, decode, what):
    """As scored_helpers.assert_scored, with what a bias adds: where a slope is below zero the keys
    that matter are the farthest, whose biases are as large as slope x context, and fp32 rounds
    such a score four times (the bias of a step, its reference taken off, a key's bias, the
    sum), each by 2^-24 of it; a slope above zero matters where it has hardly any bias."""
    ref, weight = c.expected(decode)
    reach = np.abs(np.minimum(c.slopes, 0.0)) * max(int(x) for x in c.b.seq_lens)
    if c.cache == "f32":
        size = c.score_size() + float(reach.max())
        assert_scored_f32(got, ref, weight, int(max(c.b.seq_lens)), size, what)
        return
    got = f64(got)
    score = (2.0 ** -12 + c.mods["softcap"] * 2.0 ** -21 + 4 * 2.0 ** -24 * reach)[None, :, None]
    p = 2 * 2.0 ** -8 + 2 * score
    bound = p * weight * (1 + 2.0 ** -6) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref) + 1e-30
    err = np.abs(got - ref)
    share = float((err / bound).max())
    say(what, f"worst share of the bound {share:.3f}")
    assert np.isfinite(got).all() and share <= 1.0, (what, share)


@pytest.mark.parametrize("cache,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("8bit", 128),
                                     ("8bit", 64)])
@pytest.mark.parametrize("mods", sorted(MODS))
def test_decode(cache, d, mods):
    say("decode slopes", cache, d, mods)
    for lens in ([3971], [1, 40, 700, 3001, 4097]):
        c = _call(lens, [1] * len(lens), d, cache, **MODS[mods])
        _check(c, c.decode(), True, f"{cache} {d} {mods} {len(lens)}")


@pytest.mark.parametrize("cache", ["bf16", "8bit"])
@pytest.mark.parametrize("mods", sorted(MODS))
def test_prefill(cache, mods):
    """Whole tiles, tiles that several workgroups share, and one-row sequences."""
    say("prefill slopes", cache, mods)
    for lens, new in (([3000], [150]), ([700, 2049, 33, 1500], [300, 64, 33, 1])):
        c = _call(lens, new, 128, cache, **MODS[mods])
        what = f"{cache} {mods} {len(lens)}"
        _check(c, c.prefill(), False, what)
        small = K.workspace(-(-(8 * (sum(new) // 32 + len(lens) + 1) + 16) // 256) * 256)
        _check(c, c.prefill(ws=small), False, what + ", whole tiles")


@pytest.mark.parametrize("cache", ["bf16", "8bit"])
@pytest.mark.parametrize("mods", [dict(window=150, softcap=20.0), dict(bias=True),
                                  dict(bias=True, softcap=20.0), dict(bias=True, window=150)])
def test_chunks_that_keep_their_tiles_give_the_prompts_bits(cache, mods):
    """A prompt in chunks of whole tiles gives, bit for bit, what it gives at once."""
    say("chunks", cache, mods)
    steep = "bias" in mods
    c = Call([600], [600], hq=8, hkv=2, d=128, cache=cache, **mods)
    if steep:
        c.dev_slopes = torch.from_numpy(SLOPES).cuda()
    small = K.workspace(-(-(8 * (600 // 32 + 2) + 16) // 256) * 256)
    whole = c.prefill(ws=small)
    q, at = c.q, 0
    for n in (64, 192, 128, 216):
        c.q = q[at:at + n].contiguous()
        c.sl = torch.tensor([at + n], dtype=torch.int32, device="cuda")
        c.cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        part = c.prefill(ws=small, max_seq_len=at + n)
        assert torch.equal(part.view(torch.int16), whole[at:at + n].view(torch.int16)), (at, n)
        at += n
    assert at == 600


@pytest.mark.parametrize("cache", ["bf16", "8bit"])
@pytest.mark.parametrize("mods", [dict(bias=True), dict(bias=True, window=30000)])
def test_a_biased_rows_bits_depend_on_itself(cache, mods):
    """Rows whose scores make their wavefronts move the softmax's reference leave the others of
    their tile their bits."""
    say("biased bits", cache)
    c = Call([40000], [64], hq=8, hkv=2, d=128, cache=cache, **mods)
    # biases of hundreds where they matter, and steps that leave most rows' references alone
    c.dev_slopes = torch.full((8,), -0.02, device="cuda")
    want = c.prefill()
    c.q[::2] *= 100
    got = c.prefill()
    assert not torch.equal(got[::2], want[::2])
    assert torch.equal(got[1::2].view(torch.int16), want[1::2].view(torch.int16))
