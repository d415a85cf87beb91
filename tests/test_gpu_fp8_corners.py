"""Decode and prefill over a layer in 8 bits where launches change their form: workgroups
that take splits in turn, plans of more sequences than one pass holds, scales other than
the usual one; and against the bf16 kernels on the same values."""
import numpy as np
import pytest
import torch

import paper_2608_23658_amd.kvattn as K
from oracle.paged_kv import attend, gather_kv
from tests.fp8_helpers import Dev8, assert_close, expected, fp8_batch
from tests.gpu_helpers import Dev, f64, require_gpu, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,bound", [
    ([20] * 300 + [51200] + [20] * 211, 65536),   # 50 splits, 48 workgroups: one wavefront each
    ([20] * 40 + [3000, 1025], 131072),           # four shares of a split by two wavefronts
])
def test_decode_in_turns(lens, bound, d):
    b, raw = fp8_batch(lens, [1] * len(lens), hq=8, hkv=2, d=d, seed=len(lens) + d)
    b.block_table = np.pad(b.block_table, ((0, 0), (0, bound // 16 - b.block_table.shape[1])),
                           constant_values=-1)
    say("decode fp8 in turns", len(lens), bound, d)
    out = Dev8(b, raw).decode(max_seq_len=bound)
    ref, weight = expected(b, True)
    assert_close(out, ref, weight, f"decode fp8 in turns {len(lens)}, {d}")
    long = int(np.argmax(lens))
    assert_close(out[long:long + 1], ref[long:long + 1], weight[long:long + 1], "the long one")


@pytest.mark.parametrize("chunks,hq,hkv", [
    ([(40, 1)] * 590 + [(5000, 1)] * 2 + [(90, 40)] * 20, 8, 2),   # one-row sequences shared
    ([(33, 33)] * 560, 8, 1),
    ([(20, 1)] * 530 + [(64, 0)] * 5 + [(700, 300)], 8, 8),
    ([(2100, 2100)] * 9, 8, 1),                       # few sequences, more than 512 tiles
])
def test_prefill_plans_of_many(chunks, hq, hkv):
    """More than 512 sequences, or tiles: the plan takes them in several passes."""
    chunks = [chunks[i] for i in np.random.default_rng(hq).permutation(len(chunks))]
    lens, new = [c[0] for c in chunks], [c[1] for c in chunks]
    b, raw = fp8_batch(lens, new, hq=hq, hkv=hkv, d=128, seed=len(lens))
    say("prefill fp8 of many", len(lens), sum(new), hq, hkv)
    out = Dev8(b, raw).prefill()
    assert_close(out, *expected(b, False), f"prefill fp8 of many {len(lens)} {sum(new)}")


@pytest.mark.parametrize("scale", [0.0, -0.088, 1e-42, -1e-42, 0.5])
def test_decode_scales(scale):
    """Scales of either sign and of nothing: what is masked (a block that is not there, the tail of
    a step) is minus infinity after the scale. At 0.5 scores reach some tens, and
    fp32's error in them stays below 2^-12."""
    lens, gone = [1, 63, 300, 1030, 0], {2: 3, 3: 64}
    b, raw = fp8_batch(lens, [1, 1, 1, 1, 0], hq=8, hkv=2, d=128, seed=61)
    b.q, b.scale = torch.cat([b.q, torch.ones(1, 8, 128, dtype=torch.bfloat16)]), scale
    dev = Dev8(b, raw)
    for s, j in gone.items():
        dev.bt[s, j] = -1
    say("decode fp8 scale", scale)
    out = dev.decode()
    assert (out[4] == 0).all()
    for s, L in enumerate(lens[:4]):
        k, v = gather_kv(b.kv_raw(), "bf16", b.block_table[s], L, 2, 16, 128)
        keep = np.arange(L) // 16 != gone.get(s, -1)
        k, v = k[keep], v[keep]
        q = b.q[s:s + 1].double().numpy()
        ref, weight = (attend(q, k, x, len(k) - 1, scale) for x in (v, np.abs(v)))
        assert_close(out[s:s + 1], ref, weight, f"scale {scale}, sequence {s}")


@pytest.mark.parametrize("scale", [1e-42, 0.5])
@pytest.mark.parametrize("small", [False, True])
def test_prefill_scales(scale, small):
    """The least scale, where minus infinity must not become NaN, and a large one."""
    lens, new = [1, 63, 300, 1030, 700], [1, 63, 100, 1, 130]
    b, raw = fp8_batch(lens, new, hq=8, hkv=2, d=128, seed=62)
    b.scale = scale
    ws = K.workspace(-(-(8 * (sum(new) // 32 + 6) + 16) // 256) * 256) if small else None
    say("prefill fp8 scale", scale, small)
    out = Dev8(b, raw).prefill(ws=ws)
    assert_close(out, *expected(b, False), f"prefill scale {scale}")


@pytest.mark.parametrize("decode", [True, False])
def test_as_near_to_bf16_as_their_roundings_let(decode):
    """The bf16 kernels over the layer of the same values: each is within the bound of the exact
    result, so they are within two of each other, element by element."""
    lens, new = [700, 90, 1300, 17], [1, 1, 1, 1] if decode else [200, 90, 1, 5]
    b, raw = fp8_batch(lens, new, hq=32, hkv=8, d=128, seed=14)
    dev, other = Dev8(b, raw), Dev(b)
    say("fp8 against bf16", decode)
    x, y = (f64(t.decode() if decode else t.prefill()) for t in (dev, other))
    ref, weight = expected(b, decode)
    assert_close(x, ref, weight, "8 bits")
    assert_close(y, ref, weight, "bf16")
    p = 2 * 2.0 ** -8 + 2 * 2.0 ** -12
    bound = (p * weight * (1 + 2.0 ** -7)) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref) + 1e-30
    assert (np.abs(x - y) <= 2 * bound).all()
    # Three roundings of at most 2^-8, 2^-8 / sqrt(3) in the mean square: p in the sum of p v
    # (of zero-mean v, so as large against the output as against p), p in the row
    # sum, the output; in quadrature 2^-8.
    e = [np.linalg.norm(t - ref) / np.linalg.norm(ref) for t in (x, y)]
    say("rel_l2", *(f"{t:.3e}" for t in e))
    assert max(e) <= 2.0 ** -8
