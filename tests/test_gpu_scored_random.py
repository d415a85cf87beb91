"""Seeded random calls with capped, biased and windowed scores against the fp64 oracle: lengths,
chunks, heads, caches, caps of any size, slopes of either sign, windows and workspaces drawn
together, and tables whose entries behind a window name others' blocks, which hold NaN."""
import numpy as np
import pytest
import torch

import paper_2608_23658_amd.kvattn as K
from tests.gpu_helpers import f64, require_gpu, say
from tests.scored_helpers import Call, assert_scored_f32

pytestmark = pytest.mark.gpu
EDGES = [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 1023, 1024, 1025]
HEADS = [(8, 8), (8, 4), (8, 2), (8, 1), (12, 3), (32, 8), (6, 3), (1, 1)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _draw(rng, decode):
    cache = str(rng.choice(["bf16", "8bit"] + ["f32"] * decode))
    d = 64 if cache == "f32" else 128 if not decode else int(rng.choice([64, 128]))
    hq, hkv = HEADS[rng.integers(len(HEADS))]
    B = int(rng.integers(1, 7))
    ctx = [int(rng.choice(EDGES)) if rng.random() < 0.3 else int(rng.integers(0, 1800))
           for _ in range(B)]
    new = [1 if decode or rng.random() < 0.3 else int(rng.integers(1, 260)) for _ in range(B)]
    lens = [c + n for c, n in zip(ctx, new)]
    softcap = float(rng.choice([0.0, 0.0, 5.0, 30.0, 176.0, 179.0, 1e4, 3e6]))
    window = int(rng.choice([0, 0, rng.integers(1, 50), rng.integers(50, 2000)]))
    c = Call(lens, new, hq=hq, hkv=hkv, d=d, cache=cache, seed=int(rng.integers(1 << 30)),
             q_size=float(rng.choice([1.0, 4.0])), softcap=softcap, window=window,
             bias=bool(rng.random() < 0.5))
    if c.slopes is not None:
        c.slopes = (rng.choice([-1.0, 1.0], hq) * 2.0 ** rng.uniform(-9, 3, hq)).astype(np.float32)
        c.dev_slopes = torch.from_numpy(c.slopes).cuda()
    if rng.random() < 0.2:
        c.scale = -c.scale
    what = (f"{cache} {hq}/{hkv}/{d} lens {lens} new {new} cap {softcap} window {window} "
            f"bias {c.slopes is not None}")
    say("decode" if decode else "prefill", what)
    return c, lens, new, what


def _check(c, got, decode, what):
    """As scored_helpers.assert_scored, counting what fp32 rounds of a bias (four roundings of
    slope x context where the slope is below zero) and of a cap: softcap * 2^-21 up to 177, then
    2^-19 of a score, whose size here is under 2^7."""
    ref, weight = c.expected(decode)
    top = max(int(x) for x in c.b.seq_lens)
    reach = np.zeros(c.b.num_q_heads)
    if c.slopes is not None:
        reach = np.abs(np.minimum(c.slopes, 0.0)) * top
    if c.cache == "f32":
        assert_scored_f32(got, ref, weight, top, c.score_size() + float(reach.max()), what)
        return
    cap = c.mods["softcap"]
    score = 2.0 ** -12 + min(cap, 177.0) * 2.0 ** -21 + (2.0 ** -12 if cap > 177 else 0.0)
    p = 2 * 2.0 ** -8 + 2 * (score + 4 * 2.0 ** -24 * reach)[None, :, None]
    bound = p * weight * (1 + 2.0 ** -6) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref) + 1e-30
    got = f64(got)
    share = float((np.abs(got - ref) / bound).max())
    say(f"worst share of the bound {share:.3f}")
    assert np.isfinite(got).all() and share <= 1.0, (what, share)


def _give_up(c, lens, new):
    """Blocks behind the windows become others', which hold NaN; their ids stay in the table."""
    window, gone = c.mods["window"], []
    for s, (L, n) in enumerate(zip(lens, new)):
        if window:
            gone += list(c.b.block_table[s][:max(0, L - n - window + 1) // 16])
    if gone:
        layer = c.kv.clone().view(c.b.num_blocks, -1)
        layer[torch.tensor(sorted(gone)).cuda()] = 0xff if c.cache == "8bit" else float("nan")
        c.kv = layer.view(c.kv.shape)


@pytest.mark.parametrize("seed", range(40))
def test_decode(seed):
    rng = np.random.default_rng(9000 + seed)
    c, lens, new, what = _draw(rng, True)
    _give_up(c, lens, new)
    loose = int(rng.integers(0, 3)) * 1000
    need = (c.b.max_seq_len + loose) // 16 + 1
    short = max(0, need - c.b.block_table.shape[1])
    c.b.block_table = np.pad(c.b.block_table, ((0, 0), (0, short)), constant_values=-1)
    c.set_table()
    _check(c, c.decode(max_seq_len=c.b.max_seq_len + loose), True, what)


@pytest.mark.parametrize("seed", range(40))
def test_prefill(seed):
    rng = np.random.default_rng(9500 + seed)
    c, lens, new, what = _draw(rng, False)
    _give_up(c, lens, new)
    T = sum(new)
    small = K.workspace(-(-(8 * (T // 32 + len(lens) + 1) + 16) // 256) * 256)
    _check(c, c.prefill(), False, what)
    _check(c, c.prefill(ws=small), False, what + ", whole tiles")
