"""Shared pieces of the tests of capped, biased and windowed scores: calls over either
cache, and the bound an output is held to."""
import numpy as np
import torch

import oracle
import paper_2608_23658_amd.kvattn as K
from oracle.scored import scored_attention
from tests.fp8_helpers import fp8_batch
from tests.gpu_helpers import assert_parity, f64, say
from workloads import make_batch_from_lens

MODS = {
    "cap": dict(softcap=20.0),
    "bias": dict(bias=True),
    "window": dict(window=100),
    "all": dict(softcap=5.0, bias=True, window=333),
}


class Call:
    """A batch on the device, over a cache of its own type or in 8 bits."""

    def __init__(self, lens, new, *, hq, hkv, d, cache="bf16", seed=0, q_size=4.0, softcap=0.0,
                 bias=False, window=0, scale=None):
        if cache == "8bit":
            b, raw = fp8_batch(lens, new, hq=hq, hkv=hkv, d=d, seed=seed)
            self.kv = torch.from_numpy(raw).cuda()
        else:
            b = make_batch_from_lens(lens, new, dtype=cache, num_q_heads=hq, num_kv_heads=hkv,
                                     head_dim=d, block_size=16, seed=seed)
            self.kv = b.kv_layer.cuda()
        b.q = (b.q.float() * q_size).to(b.q.dtype)       # scores of several units
        self.b, self.cache, self.q = b, cache, b.q.cuda()
        self.scale = b.scale if scale is None else scale
        self.mods = dict(softcap=softcap, window=window)
        self.slopes = None
        if bias:
            self.slopes = (2.0 ** (-8.0 * np.arange(1, hq + 1) / hq)).astype(np.float32)
            self.slopes[-1] *= -1e-3                     # one that favours far keys a little
        self.dev_slopes = None if self.slopes is None else torch.from_numpy(self.slopes).cuda()
        self.set_table()

    def set_table(self):
        self.bt = torch.from_numpy(np.ascontiguousarray(self.b.block_table)).cuda()
        self.sl = torch.from_numpy(self.b.seq_lens).cuda()
        self.cu = torch.from_numpy(self.b.cu_seqlens_q).cuda()

    def _kw(self, kw):
        return dict(dict(num_kv_heads=self.b.num_kv_heads, max_seq_len=self.b.max_seq_len,
                         scale=self.scale, slopes=self.dev_slopes, **self.mods), **kw)

    def decode(self, **kw):
        call = K.decode_scored_fp8 if self.cache == "8bit" else K.decode_scored
        return call(self.q, self.kv, self.b.num_blocks, self.bt, self.sl, **self._kw(kw))

    def prefill(self, **kw):
        call = K.prefill_chunk_scored_fp8 if self.cache == "8bit" else K.prefill_chunk_scored
        return call(self.q, self.kv, self.b.num_blocks, self.bt, self.sl, self.cu,
                    **self._kw(kw))

    def expected(self, decode):
        b = self.b
        cu = np.arange(len(b.seq_lens) + 1) if decode else b.cu_seqlens_q
        return scored_attention(b.q_raw(), b.kv_raw(), b.block_table, b.seq_lens, cu,
                                dtype=b.dtype, num_q_heads=b.num_q_heads,
                                num_kv_heads=b.num_kv_heads, head_dim=b.head_dim,
                                scale=self.scale, slopes=self.slopes, **self.mods)

    def score_size(self):
        """The largest scale * sum |q_j k_j| of a decode row and a key."""
        b, top = self.b, 0.0
        q = np.abs(oracle.storage_to_f64(b.q_raw(), b.dtype)).reshape(-1, b.num_q_heads, b.head_dim)
        for s, L in enumerate(b.seq_lens):
            k, _ = oracle.gather_kv(b.kv_raw(), b.dtype, b.block_table[s], int(L), b.num_kv_heads,
                                    16, b.head_dim)
            k = np.repeat(np.abs(k), b.num_q_heads // b.num_kv_heads, 1)
            top = max(top, float(np.einsum("hd,thd->th", q[s], k).max()) * abs(self.scale))
        return top

    def check(self, got, decode, what):
        assert_scored(got, *self.expected(decode), self.cache, self.mods["softcap"], what)


def assert_scored_f32(got, ref, weight, keys, size, what):
    """fp32 where scores are large: a dot product of 64 terms is off by at most 64 roundings of
    the sum of their sizes (at most ``size`` with the scale), the scale, the cap and the
    maximum by six more; p is off by as much of itself and two units, in both sums, which
    add at most ``keys`` terms; the quotient is two more."""
    got = f64(got)
    e = 2.0 ** -24
    bound = weight * 2 * ((64 + 6) * e * size + 2 * e + (keys + 2) * e) * 1.01 + 1e-37
    err = np.abs(got - ref)
    say(what, f"worst share of the bound {float((err / bound).max()):.3f}")
    assert np.isfinite(got).all() and (err <= bound).all(), what


def assert_scored(got, ref, weight, cache, softcap, what):
    """Every element within what roundings allow. In bf16 p is rounded (at most 2^-8 of
    itself) in the sum of p v and in the sum of p alike; a score that is off by e makes p off by
    e of itself, twice again: fp32's error of a dot product and of its bias, under 2^-12 for
    scores that matter here (within 40 of a row's largest), and the cap's 2^-21 of it; the
    output is rounded to bf16. fp32 by the framework's bound."""
    got = f64(got) if isinstance(got, torch.Tensor) else got
    if cache == "f32":
        assert_parity(got, ref, "f32", what)
        return
    p = 2 * 2.0 ** -8 + 2 * (2.0 ** -12 + softcap * 2.0 ** -21)
    bound = (p * weight * (1 + 2.0 ** -7)) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref) + 1e-30
    err = np.abs(got - ref)
    assert np.isfinite(got).all(), what
    rel = float(np.linalg.norm(err) / max(np.linalg.norm(ref), 1e-30))
    say(what, f"worst share of the bound {float((err / bound).max()):.3f} rel_l2 {rel:.3e}")
    assert (err <= bound).all(), (what, float((err / bound).max()))
    assert rel <= 1e-2, (what, rel)
