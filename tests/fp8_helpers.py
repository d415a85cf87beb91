"""Shared pieces of the GPU tests of the layer in 8 bits: batches whose blocks have
scales of their own, calls, and the bound an output is held to."""
import numpy as np
import torch

import paper_2608_23658_amd.kvattn as K
from oracle import fp8
from tests.gpu_helpers import f64, oracle_decode, oracle_prefill, say
from workloads import make_batch_from_lens


def u16(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


def bf16_tensor(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16)


def fp8_batch(lens, q_lens, *, hq, hkv, d, seed, spread=2):
    """A batch whose layer holds values that 8 bits hold exactly (``b.kv_layer``, bf16, for the
    oracle) and its bytes; each tile is scaled by a power of two of its own. Slots
    past a sequence's end and free blocks are NaN in both."""
    b = make_batch_from_lens(lens, q_lens, dtype="bf16", num_q_heads=hq, num_kv_heads=hkv,
                             head_dim=d, block_size=16, seed=seed)
    rng = np.random.default_rng(seed)
    x = b.kv_layer.view(b.num_blocks, 2, hkv, 16 * d)
    by = torch.from_numpy(np.exp2(rng.integers(-spread, spread + 1, (b.num_blocks, 2, hkv, 1))))
    by[:, 0] = by[:, 0].clamp(max=1.0)          # keys: scores stay those of N(0, 1) at most
    raw = fp8.from_bf16_layer(u16((x * by).to(torch.bfloat16).reshape(-1)), hkv, d)
    b.kv_layer = bf16_tensor(fp8.to_bf16_layer(raw, hkv, d))
    return b, raw


class Dev8:
    def __init__(self, b, raw):
        self.b = b
        self.q, self.kv = b.q.cuda(), torch.from_numpy(raw).cuda()
        self.bt = torch.from_numpy(b.block_table).cuda()
        self.sl = torch.from_numpy(b.seq_lens).cuda()
        self.cu = torch.from_numpy(b.cu_seqlens_q).cuda()

    def decode(self, **kw):
        b = self.b
        kw = dict(dict(max_seq_len=b.max_seq_len), **kw)
        return K.decode_fp8(self.q, self.kv, b.num_blocks, self.bt, self.sl,
                            num_kv_heads=b.num_kv_heads, scale=b.scale, **kw)

    def prefill(self, **kw):
        b = self.b
        kw = dict(dict(max_seq_len=b.max_seq_len), **kw)
        return K.prefill_chunk_fp8(self.q, self.kv, b.num_blocks, self.bt, self.sl, self.cu,
                                   num_kv_heads=b.num_kv_heads, scale=b.scale, **kw)


def expected(b, decode):
    """The oracle's output, and sum p |v| (its output for |V|)."""
    run = oracle_decode if decode else oracle_prefill
    ref = run(b)
    keep = b.kv_layer
    lay = keep.clone().view(b.num_blocks, 2, b.num_kv_heads, -1)
    lay[:, 1] = lay[:, 1].abs()
    b.kv_layer = lay.view(-1)
    weight = run(b)
    b.kv_layer = keep
    return ref, weight


def assert_close(got, ref, weight, what):
    """Every element within what roundings allow. p is rounded to bf16 (at most 2^-8 of
    itself) in the sum of p v and in the sum of p alike: 2 * 2^-8 of sum p |v| / sum p;
    scores have fp32's error, under 2^-12 of p for the scores here, twice again;
    the output is rounded to bf16: 2^-8 of its value, itself off by the rest. And the
    2-norm is within the framework's 1e-2."""
    got = f64(got) if isinstance(got, torch.Tensor) else got
    p = 2 * 2.0 ** -8 + 2 * 2.0 ** -12
    bound = (p * weight * (1 + 2.0 ** -7)) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref) + 1e-30
    err = np.abs(got - ref)
    assert np.isfinite(got).all(), what
    rel = float(np.linalg.norm(err) / max(np.linalg.norm(ref), 1e-30))
    say(what, f"worst share of the bound {float((err / bound).max()):.3f} rel_l2 {rel:.3e}")
    assert (err <= bound).all(), (what, float((err / bound).max()))
    assert rel <= 1e-2, (what, rel)
