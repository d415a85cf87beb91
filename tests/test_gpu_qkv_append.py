"""Norm, rotation and cache write in one call, against the oracle.

A value of q or k is computed in fp32 and rounded once. Its fp32 error is at most that of a
sum of 128 squares (34 roundings one after another, halved by the root), the root (2), three
products and the rotation's three: 2^-24 * 27, under 2^-19 of the size of the terms it sums."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_23658_amd.kvattn as K
from oracle.qkv import norm_rope, rope_table
from tests.gpu_helpers import require_gpu, say

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
FP32_ERROR = 2.0 ** -19
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def raw(t):
    t = t.detach().cpu().contiguous()
    return t.view(torch.int16).numpy().view(np.uint16) if t.dtype == torch.bfloat16 else t.numpy()


def f64(t):
    return t.detach().double().cpu().numpy()


class Rows:
    """A call's inputs: q, k, v as parts of one fused buffer, or apart."""

    def __init__(self, T, hq, hkv, d, dtype, *, seed=0, norm=(True, True), rot=None, axes=1,
                 sections=None, interleaved=False, max_pos=5000, fused=True, nb=None, slots=None):
        g = torch.Generator().manual_seed(seed)
        self.T, self.hq, self.hkv, self.d, self.dtype = T, hq, hkv, d, dtype
        size = torch.exp2(torch.randint(-4, 5, (T, hq + 2 * hkv, 1), generator=g).float())
        x = (torch.randn(T, hq + 2 * hkv, d, generator=g) * size).to(DT[dtype]).cuda()
        parts = x.split((hq, hkv, hkv), 1)
        self.q, self.k, self.v = parts if fused else [p.contiguous() for p in parts]
        w = [(1 + 0.3 * torch.randn(d, generator=g)).to(DT[dtype]).cuda() for _ in range(2)]
        self.wq, self.wk = (w[i] if norm[i] else None for i in range(2))
        self.rot, self.interleaved, self.sections = rot, interleaved, sections
        self.table = self.pos = None
        if rot:
            self.table = rope_table(max_pos, rot)
            pos = torch.randint(0, max_pos, (axes, T), generator=g).to(torch.int32)
            self.pos = pos if sections else pos[0]
        rng = np.random.default_rng(seed)
        self.nb = T // 16 + 5 if nb is None else nb
        if slots is None:
            slots = rng.permutation(self.nb * 16)[:T]
        self.slots = np.asarray(slots, np.int32)
        layer = torch.randn(self.nb * 2 * hkv * 16 * d, generator=g).to(DT[dtype])
        layer[::5] = float("nan")
        self.layer = layer.cuda()

    def call(self, fn=None, **kw):
        args = dict(q_weight=self.wq, k_weight=self.wk, eps=EPS, interleaved=self.interleaved)
        if self.rot:
            args.update(rope_table=torch.from_numpy(self.table).cuda(), positions=self.pos.cuda(),
                        sections=self.sections)
        args.update(kw)
        return (fn or K.qkv_append)(self.q, self.k, self.v, torch.from_numpy(self.slots).cuda(),
                                    self.layer, self.nb, **args)

    def expected(self, which):
        x, w = (self.q, self.wq) if which == "q" else (self.k, self.wk)
        return norm_rope(f64(x), weight=None if w is None else f64(w), eps=EPS, table=self.table,
                         positions=None if self.pos is None else self.pos.numpy(),
                         sections=self.sections, interleaved=self.interleaved)


def assert_rounded(got, ref, size, dtype, what):
    bad = np.isnan(ref)
    assert np.array_equal(np.isnan(got), bad), what
    tol = FP32_ERROR * size * (1 + HALF_STEP[dtype]) + HALF_STEP[dtype] * np.abs(ref)
    err = np.abs(got - ref)[~bad]
    tol = tol[~bad] + 1e-37
    say(what, f"worst share of the bound {float((err / tol).max()) if err.size else 0:.3f}")
    assert (err <= tol).all(), (what, float((err / tol).max()))


def assert_layer(r, before, after, what):
    """v bit for bit, k within its rounding, every other element as it was."""
    want = oracle.kv_append(before, np.zeros((r.T, r.hkv, r.d), before.dtype), raw(r.v), r.slots,
                            dtype=r.dtype, num_kv_heads=r.hkv, head_dim=r.d, block_size=16)
    mark = oracle.kv_append(np.zeros_like(before), np.ones((r.T, r.hkv, r.d), before.dtype),
                            np.zeros((r.T, r.hkv, r.d), before.dtype), r.slots, dtype=r.dtype,
                            num_kv_heads=r.hkv, head_dim=r.d, block_size=16)
    is_k = mark.reshape(-1) != 0
    same = after.reshape(-1).view(np.uint8).reshape(-1, after.itemsize) == \
        want.reshape(-1).view(np.uint8).reshape(-1, after.itemsize)
    assert same.all(1)[~is_k].all(), what
    ref, size = r.expected("k")
    vec, j = 16 // after.itemsize, np.arange(r.d)
    lay = oracle.storage_to_f64(after, r.dtype).reshape(-1, 2, r.hkv, 16 * r.d)
    live = (r.slots >= 0) & (r.slots < r.nb * 16)
    b, s = r.slots[live] // 16, r.slots[live] % 16
    got = np.stack([lay[b[:, None], 0, g, (j // vec * 16 + s[:, None]) * vec + j % vec]
                    for g in range(r.hkv)], 1)
    assert_rounded(got, ref[live], size[live], r.dtype, what + " k")


def check(r, what, **kw):
    say("qkv append", what, r.T, r.hq, r.hkv, r.d, r.dtype)
    before = raw(r.layer).copy()
    ref, size = r.expected("q")
    out = r.call(**kw)
    torch.cuda.synchronize()
    assert_layer(r, before, raw(r.layer), what)
    assert_rounded(f64(out), ref, size, r.dtype, what + " q")
    return out


SHAPES = [("bf16", 8, 2, 128), ("bf16", 3, 1, 64), ("f32", 4, 2, 128), ("f32", 6, 3, 64)]


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("share", [None, 1, 2, 4])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotations(dtype, hq, hkv, d, share, interleaved):
    """No rotation, and all, half and a quarter (32 dims at least) of the dims."""
    rot = share and max(32, d // share)
    check(Rows(37, hq, hkv, d, dtype, rot=rot, interleaved=interleaved), f"rot {rot}")


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("T", [1, 15, 16, 17, 333])
@pytest.mark.parametrize("fused", [True, False])
def test_lengths(dtype, hq, hkv, d, T, fused):
    check(Rows(T, hq, hkv, d, dtype, rot=d, fused=fused, seed=T), f"T {T} fused {fused}")


@pytest.mark.parametrize("norm", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("rot", [None, 64])
def test_norms_apart(norm, rot):
    check(Rows(21, 4, 4, 64, "bf16", norm=norm, rot=rot), f"norm {norm}")


@pytest.mark.parametrize("dtype,d,rot", [("bf16", 128, 128), ("bf16", 128, 32), ("bf16", 64, 64),
                                         ("f32", 64, 32), ("f32", 128, 128)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("cut", [(1, 1), (3, -2, 2), (0, 5, -1, 0), (8, 4, -4)])
def test_axes(dtype, d, rot, interleaved, cut):
    """Sections that end inside a register's run of pairs, at its end, and empty ones."""
    sections = [abs(c) for c in cut]
    sections[-1] = rot // 2 - sum(sections[:-1])
    check(Rows(40, 3, 2, d, dtype, rot=rot, axes=len(cut), sections=sections,
               interleaved=interleaved), f"sections {sections}")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("T,start", [(16, 0), (64, 5), (1, 15), (700, 0), (701, 9)])
def test_tokens_in_order(dtype, d, T, start):
    """A chunk's tokens: whole blocks in order, and runs that cross a block's border."""
    nb = (T + start) // 16 + 3
    perm = np.random.default_rng(T).permutation(nb)
    t = np.arange(start, start + T)
    check(Rows(T, 8, 2, d, dtype, rot=d, nb=nb, slots=perm[t // 16] * 16 + t % 16), "in order")


def test_many_heads_and_tokens():
    """Sizes at which a wavefront takes several heads."""
    T = 2100
    t = np.arange(T) + 3
    check(Rows(T, 64, 8, 64, "bf16", rot=64, nb=T // 16 + 2, slots=t), "many")


def test_padding_and_slots_outside():
    """Tokens without a slot: nothing is written for them, their q is."""
    r = Rows(50, 4, 2, 64, "bf16", rot=64)
    r.slots[[0, 7, 49]] = -1
    r.slots[[3, 20]] = [r.nb * 16, 2 ** 31 - 1]
    r.slots[21] = -2 ** 31
    check(r, "padding")


def test_positions_outside_the_table():
    r = Rows(20, 2, 2, 64, "bf16", rot=32, max_pos=100)
    r.pos[[1, 4, 5]] = torch.tensor([-1, 100, 2 ** 31 - 1], dtype=torch.int32)
    check(r, "positions outside")


def test_zero_rows_and_special_values():
    r = Rows(20, 2, 1, 64, "f32", rot=64)
    r.q[0], r.k[1], r.v[2, 0, :2] = 0, 0, torch.tensor([float("nan"), float("inf")])
    check(r, "zeros")


def test_in_place_and_out():
    r = Rows(33, 4, 2, 128, "bf16", rot=128, fused=False)
    ref, size = r.expected("q")
    out = r.call(out=r.q)
    assert out.data_ptr() == r.q.data_ptr()
    torch.cuda.synchronize()
    assert_rounded(f64(out), ref, size, "bf16", "in place")
    r = Rows(33, 4, 2, 128, "bf16", rot=128)
    out = torch.full((33, 4, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    assert check(r, "out", out=out) is out


def test_tokens_far_apart():
    """Rows 2^31 elements from the first and beyond: offsets in 64 bits."""
    T, gap = 5, 600_000_000
    buf = torch.empty((T - 1) * gap + 4 * 64, dtype=torch.bfloat16, device="cuda")
    view = buf.as_strided((T, 4, 64), (gap, 64, 1))
    r = Rows(T, 2, 1, 64, "bf16", rot=64)
    view[:, :2], view[:, 2:3], view[:, 3:] = r.q, r.k, r.v
    r.q, r.k, r.v = view.split((2, 1, 1), 1)
    check(r, "far apart")


def test_a_layer_past_4_gib():
    """Slots whose block lies beyond 2^32 bytes."""
    r = Rows(40, 2, 8, 128, "bf16", rot=128, nb=40)
    nb = 80_000                                   # 5.2 GB
    big = torch.zeros(nb * 2 * 8 * 16 * 128, dtype=torch.bfloat16, device="cuda")
    blocks = np.random.default_rng(0).permutation(40)
    small, r.layer, r.nb = r.layer, big, nb
    slots = r.slots.copy()
    r.slots = ((nb - 1 - blocks[slots // 16]) * 16 + slots % 16).astype(np.int32)
    out = r.call()
    high = big.view(nb, -1)[nb - 40:].cpu()
    assert not big.view(nb, -1)[:nb - 40].any()
    r.layer, r.nb = torch.zeros_like(small), 40
    r.slots = (r.slots - (nb - 40) * 16).astype(np.int32)
    again = r.call()
    assert torch.equal(raw_t(out), raw_t(again))
    assert torch.equal(raw_t(high.reshape(-1)), raw_t(r.layer.cpu()))


def raw_t(t):
    return t.contiguous().view(torch.int16)


def test_same_bits_in_any_batch():
    """A token's row does not depend on the call's others, or on how many heads a wavefront
    takes."""
    big = Rows(1500, 32, 8, 128, "bf16", rot=128)
    out = big.call()
    at = slice(700, 709)
    layer = torch.zeros_like(big.layer)
    few = K.qkv_append(big.q[at], big.k[at], big.v[at], torch.from_numpy(big.slots[at]).cuda(),
                       layer, big.nb, positions=big.pos[at].cuda(), q_weight=big.wq,
                       k_weight=big.wk, eps=EPS, rope_table=torch.from_numpy(big.table).cuda())
    torch.cuda.synchronize()
    assert torch.equal(raw_t(few), raw_t(out[at]))
    written = raw_t(layer) != 0
    assert torch.equal(raw_t(layer)[written], raw_t(big.layer)[written])


def _patterns(T, nb, seed):
    """Slot lists that mix runs in order with single tokens in every way."""
    r = np.random.default_rng(seed)
    yield "backwards", np.arange(T)[::-1] + 3
    a, b = np.arange((T + 1) // 2) + 5, np.arange(T // 2) + 16 * (nb // 2) + 11
    two = np.empty(T, np.int64)
    two[0::2], two[1::2] = a, b
    yield "two sequences by turns", two
    yield "every other slot", np.arange(T) * 2 + 1
    runs, free = [], list(r.permutation(nb))
    while sum(map(len, runs)) < T:           # parts of blocks, 1 to 16 tokens long
        lo = int(r.integers(0, 16))
        n = int(r.integers(1, 17 - lo))
        at = free.pop() * 16 + lo
        runs.append(np.arange(at, at + n))
    parts = np.concatenate(runs)[:T]
    yield "parts of blocks", parts
    holes = parts.copy()
    holes[r.random(T) < 0.2] = -1
    holes[r.random(T) < 0.1] = nb * 16 + 3
    yield "parts of blocks with holes", holes
    swapped = parts.copy()
    i = r.integers(0, T - 1, T // 8)
    for j in i:
        swapped[[j, j + 1]] = swapped[[j + 1, j]]
    yield "parts of blocks, some swapped", swapped


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("T", [17, 33, 130, 515])
def test_slot_patterns(dtype, d, T):
    nb = T + 10
    for what, slots in _patterns(T, nb, T):
        check(Rows(T, 4, 2, d, dtype, rot=d // 2, nb=nb, slots=slots), what)
