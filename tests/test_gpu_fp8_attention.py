"""Decode and chunked prefill over a layer in 8 bits against the fp64 oracle run on the
same values."""
import numpy as np
import pytest
import torch

import paper_2608_23658_amd.kvattn as K
from oracle import fp8
from tests.fp8_helpers import Dev8, assert_close, bf16_tensor, expected, fp8_batch, u16
from tests.gpu_helpers import require_gpu, say

pytestmark = pytest.mark.gpu
RAGGED = [1, 15, 16, 17, 63, 64, 65, 511, 512, 513, 1023, 1024, 1025, 1500, 2049, 4097]
HEADS = [(32, 8, 128), (8, 8, 128), (16, 8, 128), (64, 8, 128), (12, 3, 128), (8, 1, 128),
         (8, 2, 64), (4, 4, 64), (8, 4, 64), (16, 2, 64), (64, 8, 64)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_decode_ragged(hq, hkv, d):
    b, raw = fp8_batch(RAGGED, [1] * len(RAGGED), hq=hq, hkv=hkv, d=d, seed=hq + d)
    say("decode fp8", hq, hkv, d)
    out = Dev8(b, raw).decode()
    assert_close(out, *expected(b, True), f"decode fp8 {hq}/{hkv}/{d}")


@pytest.mark.parametrize("lens,bound", [
    ([3971], 3971),                    # a workgroup per wavefront
    ([37], 4096), ([1], 1), ([64, 1, 63], 64),
    ([5000, 1, 9000, 700], 9000),
    ([20] * 40 + [300], 131072),       # far more workgroups than work
    ([200] * 300, 200),
])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_by_launch(lens, bound, d):
    b, raw = fp8_batch(lens, [1] * len(lens), hq=16, hkv=2, d=d, seed=len(lens) + bound)
    b.block_table = np.pad(b.block_table, ((0, 0), (0, bound // 16 + 1 - b.block_table.shape[1])),
                           constant_values=-1) if b.block_table.shape[1] * 16 < bound else b.block_table
    say("decode fp8", len(lens), bound, d)
    out = Dev8(b, raw).decode(max_seq_len=bound)
    assert_close(out, *expected(b, True), f"decode fp8 {len(lens)} under {bound}, {d}")


@pytest.mark.parametrize("hq,hkv,d", [(12, 3, 128), (32, 8, 128), (8, 2, 64), (40, 5, 64)])
def test_decode_many(hq, hkv, d):
    """Enough workgroups that heads are placed by XCD, with some left over."""
    lens = np.random.default_rng(hkv).integers(1, 1500, 117).tolist() + [0, 3000]
    b, raw = fp8_batch(lens, [0 if n == 0 else 1 for n in lens], hq=hq, hkv=hkv, d=d, seed=hkv)
    dev = Dev8(b, raw)
    i = lens.index(0)                      # decode has a row for the empty sequence too
    q = torch.cat([b.q[:i], torch.ones(1, hq, d, dtype=torch.bfloat16), b.q[i:]])
    b.q, dev.q = q, q.cuda()
    say("decode fp8 many", hq, hkv, d)
    assert_close(dev.decode(), *expected(b, True), f"decode fp8 many {hq}/{hkv}/{d}")


@pytest.mark.parametrize("hq,hkv", [(32, 8), (8, 8), (16, 8), (64, 8), (12, 3)])
def test_prefill_ragged(hq, hkv):
    lens = [1, 16, 17, 64, 65, 130, 300, 700, 1025]
    new = [1, 16, 3, 64, 1, 130, 100, 1, 257]
    b, raw = fp8_batch(lens, new, hq=hq, hkv=hkv, d=128, seed=hq)
    say("prefill fp8", hq, hkv)
    out = Dev8(b, raw).prefill()
    assert_close(out, *expected(b, False), f"prefill fp8 {hq}/{hkv}")


@pytest.mark.parametrize("lens,new,hq,hkv", [
    ([1], [1], 8, 1), ([33], [33], 8, 1), ([128], [64], 8, 2), ([200], [7], 32, 8),
    ([3000], [1], 16, 2),               # one row alone
    ([6150], [201], 8, 2),              # tiles shared by several workgroups
    ([2500, 1700, 1200], [1, 1, 300], 8, 1),
    ([40] * 30, [40] * 30, 8, 8),
    ([64, 64], [0, 64], 8, 2),          # a sequence without new rows
    ([300] * 5 + [1100] * 3, [1] * 5 + [2] * 3, 32, 8),
])
@pytest.mark.parametrize("small", [False, True])
def test_prefill_by_plan(lens, new, hq, hkv, small):
    b, raw = fp8_batch(lens, new, hq=hq, hkv=hkv, d=128, seed=sum(lens) + hq)
    say("prefill fp8", lens[:4], new[:4], hq, hkv, "small workspace" if small else "")
    T = sum(new)
    ws = None
    if small:
        ws = K.workspace(-(-(8 * (T // 32 + len(lens) + 1) + 16) // 256) * 256)
    out = Dev8(b, raw).prefill(ws=ws)
    assert_close(out, *expected(b, False), f"prefill fp8 {len(lens)} {T}")


def test_values_pass_through_exactly():
    """With one token the output is its V, bit for bit: every code at exponents from the
    least to the largest."""
    d, n = 128, 64
    rng = np.random.default_rng(1)
    bb = fp8.block_bytes(1, d)
    raw = np.full((n, bb), 0x7F, np.uint8)
    lay = fp8.Layer(raw.reshape(-1), 1, d)
    exps = np.linspace(10, 246, n).astype(int)
    for b in range(n):
        for kind in range(2):
            lay.set_exp(b, kind, 0, int(exps[b]) if kind else 120)
        c = rng.integers(0, 254, (2, d))
        c = np.where(c >= 127, c + 1, c).astype(np.uint8)
        lay.tile(b, 0, 0)[fp8.place(0, 0, np.arange(d))] = c[0]
        lay.tile(b, 1, 0)[fp8.place(1, 0, np.arange(d))] = c[1]
    want = np.stack([lay.values(b, 1, 0)[0] for b in range(n)]).astype(np.float32)
    q = torch.randn(n, 4, d).to(torch.bfloat16).cuda()
    kv = torch.from_numpy(lay.raw.reshape(-1)).cuda()
    bt = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].contiguous()
    sl = torch.ones(n, dtype=torch.int32, device="cuda")
    cu = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    want = np.repeat(want[:, None], 4, 1)
    say("fp8 one token")
    kw = dict(num_kv_heads=1, max_seq_len=1)
    small = K.workspace(-(-(8 * (n // 32 + n + 1) + 16) // 256) * 256)   # every row a tile
    for out in (K.decode_fp8(q, kv, n, bt, sl, **kw),
                K.prefill_chunk_fp8(q, kv, n, bt, sl, cu, **kw),
                K.prefill_chunk_fp8(q, kv, n, bt, sl, cu, ws=small, **kw)):
        assert np.array_equal(out.float().cpu().numpy(), want)


@pytest.mark.parametrize("j", [0, 517, 1499])
@pytest.mark.parametrize("rows", [1, 70])
def test_one_key_takes_all(j, rows):
    """A key so large that all other weights vanish: the output is that token's V, bit for
    bit, so every index on the way is right."""
    L, hq, hkv, d = 1500, 8, 2, 128
    b, raw = fp8_batch([L], [rows], hq=hq, hkv=hkv, d=d, seed=j + rows)
    j = min(j, L - rows)                    # seen by every row
    b.q[:, :, 0] = 16.0
    lay = fp8.Layer(raw, hkv, d)
    blk, r = int(b.block_table[0, j // 16]), j % 16
    for g in range(hkv):
        lay.set_exp(blk, 0, g, 127)
        lay.tile(blk, 0, g)[:] = 0
        lay.tile(blk, 0, g)[fp8.place(0, r, 0)] = fp8.encode(192.0)
    raw = lay.raw.reshape(-1)
    say("fp8 one key", j, rows)
    dev = Dev8(b, raw)
    out = (dev.decode() if rows == 1 else dev.prefill()).float().cpu().numpy()
    for g in range(hkv):
        want = lay.values(blk, 1, g)[r].astype(np.float32)
        assert (out[:, g * 4:(g + 1) * 4] == want).all()


def test_empty_sequences_and_rows_behind_the_last():
    b, raw = fp8_batch([1, 0, 40, 0], [1, 0, 1, 0], hq=8, hkv=2, d=128, seed=8)
    dev = Dev8(b, raw)
    dev.q = torch.randn(4, 8, 128).to(torch.bfloat16).cuda()
    say("decode fp8 empty")
    out = dev.decode()
    assert (out[1] == 0).all() and (out[3] == 0).all() and torch.isfinite(out.float()).all()
    # a padded batch: rows past cu[num_seqs] stay as they were
    b, raw = fp8_batch([100, 70], [40, 1], hq=8, hkv=2, d=128, seed=9)
    dev = Dev8(b, raw)
    ref = dev.prefill()
    dev.q = torch.cat([dev.q, torch.full((9, 8, 128), float("nan"), dtype=torch.bfloat16,
                                         device="cuda")])
    keep = torch.full((50, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    say("prefill fp8 padded")
    out = dev.prefill(out=keep)
    assert torch.equal(out[:41], ref) and (out[41:] == 7).all()


@pytest.mark.parametrize("decode", [True, False])
def test_bad_ids_contribute_nothing(decode):
    """A block id outside the layer removes its tokens: the same as a sequence whose
    scores there are minus infinity."""
    lens = [300, 200, 130]
    new = [1, 1, 1] if decode else [100, 50, 7]
    b, raw = fp8_batch(lens, new, hq=8, hkv=2, d=128, seed=21)
    dev = Dev8(b, raw)
    bt = b.block_table.copy()
    gone = {0: [3], 1: [0, 5], 2: [8]}
    bt[0, 3], bt[1, 0], bt[1, 5], bt[2, 8] = b.num_blocks + 1000, -5, 1 << 30, b.num_blocks
    dev.bt = torch.from_numpy(bt).cuda()
    say("fp8 bad ids", decode)
    got = (dev.decode() if decode else dev.prefill()).double().cpu()
    k, v = _contig(b)
    for s in range(3):
        L, n, r0 = lens[s], new[s], int(b.cu_seqlens_q[s])
        t = torch.arange(L)
        keep = t[None] <= torch.arange(L - n, L)[:, None]
        for j in gone[s]:
            keep &= ~((t >= 16 * j) & (t < 16 * j + 16))[None]
        q = b.q[r0:r0 + n].double().view(n, 2, 4, 128)
        sc = torch.einsum("nghd,lgd->nghl", q, k[s]) * b.scale
        sc = sc.masked_fill(~keep[:, None, None, :], -float("inf"))
        p = torch.softmax(sc, -1).nan_to_num(0.0)          # a row that sees nothing: zeros
        ref = torch.einsum("nghl,lgd->nghd", p, v[s]).reshape(n, 8, 128)
        w = torch.einsum("nghl,lgd->nghd", p, v[s].abs()).reshape(n, 8, 128)
        assert_close(got[r0:r0 + n].numpy(), ref.numpy(), w.numpy(), f"bad ids {s}")


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("byte", [0, 127, 255])
def test_blocks_that_nobody_wrote(decode, byte):
    """What never-written blocks hold (block 0 among them), exponents outside 10 .. 246 too,
    does not reach an output: sequences that end inside a step, and entries of -1."""
    lens = [1, 17, 40, 300, 70]
    new = [1] * 5 if decode else [1, 17, 33, 100, 2]
    b, raw = fp8_batch(lens, new, hq=8, hkv=2, d=128, seed=31)
    bb = fp8.block_bytes(2, 128)
    at = 2 * 2 * 16 * 128
    lay = np.concatenate([np.full((1, bb), byte, np.uint8), raw.reshape(-1, bb)])
    free = np.setdiff1d(np.arange(b.num_blocks), b.block_table[b.block_table >= 0])
    lay[1 + free] = byte
    lay[:, at + 4:] = byte                               # the padding
    dev, clean = Dev8(b, lay.reshape(-1)), Dev8(b, raw)
    bt = b.block_table.copy()
    bt[3, 4] = -1
    clean.bt = torch.from_numpy(bt).cuda()
    dev.bt = torch.from_numpy(np.where(bt >= 0, bt + 1, -1).astype(np.int32)).cuda()
    say("fp8 unwritten blocks", decode, byte)
    small = K.workspace(-(-(8 * (sum(new) // 32 + 6) + 16) // 256) * 256)
    b.num_blocks += 1
    got = [dev.decode()] if decode else [dev.prefill(), dev.prefill(ws=small)]
    b.num_blocks -= 1
    want = [clean.decode()] if decode else [clean.prefill(), clean.prefill(ws=small)]
    for x, y in zip(got, want):
        assert torch.isfinite(x.float()).all()
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


@pytest.mark.parametrize("decode", [True, False])
def test_nan_stays_in_its_sequence(decode):
    """NaN in q, in K and in V of some sequences: the others' bits do not change, a row that sees
    one is NaN, and a NaN in K of a chunk's last token leaves the earlier rows alone."""
    lens = [300, 41, 130, 1100, 16]
    new = [1] * 5 if decode else [100, 41, 7, 1, 16]
    b, raw = fp8_batch(lens, new, hq=8, hkv=2, d=128, seed=77)
    clean = Dev8(b, raw)
    lay = fp8.Layer(raw.copy(), 2, 128)
    blk = int(b.block_table[0, 299 // 16])
    lay.tile(blk, 0, 0)[fp8.place(0, 299 % 16, 5)] = 0x7F     # K of the last token of 0, head 0
    blk = int(b.block_table[2, 3])
    lay.tile(blk, 1, 1)[fp8.place(1, 2, 64)] = 0xFF           # V of token 50 of 2, head 1
    dev = Dev8(b, lay.raw.reshape(-1))
    dev.q[-1, 3] = float("nan")                               # the last row of 4, one head
    say("fp8 nan", decode)
    x, y = (d.decode() if decode else d.prefill() for d in (dev, clean))
    want = torch.zeros(x.shape, dtype=torch.bool, device="cuda")
    at = [int(i) for i in b.cu_seqlens_q]
    want[at[1] - 1, :4] = True
    want[at[2]:at[3], 4:, 64] = True
    want[-1, 3] = True
    assert torch.equal(torch.isnan(x.float()), want)
    assert torch.equal(x.view(torch.int16)[~want], y.view(torch.int16)[~want])


def _contig(b):
    x = b.kv_layer.double().view(b.num_blocks, 2, b.num_kv_heads, -1)
    ks, vs = [], []
    for s, L in enumerate(b.seq_lens):
        ids = torch.from_numpy(b.block_table[s, :-(-int(L) // 16)].astype(np.int64))
        d = b.head_dim
        k = x[ids, 0].view(len(ids), b.num_kv_heads, d // 8, 16, 8).permute(0, 3, 1, 2, 4)
        v = x[ids, 1].view(len(ids), b.num_kv_heads, d, 16).permute(0, 3, 1, 2)
        ks.append(k.reshape(-1, b.num_kv_heads, d)[:int(L)])
        vs.append(v.reshape(-1, b.num_kv_heads, d)[:int(L)])
    return ks, vs


def test_all_ids_bad_gives_zeros():
    b, raw = fp8_batch([100, 3000], [1, 1], hq=8, hkv=2, d=128, seed=4)
    dev = Dev8(b, raw)
    dev.bt = torch.full_like(dev.bt, -1)
    say("fp8 all ids bad")
    assert (dev.decode() == 0).all() and (dev.prefill() == 0).all()


def test_block_order_and_repeats_do_not_change_bits():
    """Another layout of the same blocks, the same call again, and a workspace with
    room for one partial per split: the same bits."""
    b, raw = fp8_batch(RAGGED, [1] * len(RAGGED), hq=32, hkv=8, d=128, seed=5)
    bb = fp8.block_bytes(8, 128)
    perm = np.random.default_rng(2).permutation(b.num_blocks)
    moved = np.empty_like(raw).reshape(-1, bb)
    moved[perm] = raw.reshape(-1, bb)
    dev, dev2 = Dev8(b, raw), Dev8(b, moved.reshape(-1))
    dev2.bt = torch.from_numpy(np.where(b.block_table >= 0, perm[b.block_table], -1).astype(np.int32)).cuda()
    say("decode fp8 permuted")
    a = dev.decode()
    n = len(RAGGED) * 32 * -(-4097 // 1024)
    small = K.workspace(-(-n * 128 * 4 // 256) * 256 + -(-n * 8 // 256) * 256)
    for o in (dev2.decode(), dev.decode(), dev.decode(ws=small)):
        assert torch.equal(a.view(torch.int16), o.view(torch.int16))
    one, raw1 = fp8_batch([3971], [1], hq=32, hkv=8, d=128, seed=6)
    d1 = Dev8(one, raw1)
    n = 32 * 4
    small = K.workspace(n * 128 * 4 + n * 8)
    assert torch.equal(d1.decode(), d1.decode(ws=small))   # spread or not


def test_close_to_the_bf16_layer_of_the_same_values():
    b, raw = fp8_batch([700, 90, 1300], [1, 1, 1], hq=32, hkv=8, d=128, seed=14)
    dev = Dev8(b, raw)
    say("fp8 against bf16")
    other = K.decode(dev.q, b.kv_layer.cuda(), b.num_blocks, dev.bt, dev.sl, num_kv_heads=8,
                     max_seq_len=1300, scale=b.scale)
    # two orders of the same fp32 sums, one rounding to bf16 each
    assert torch.allclose(dev.decode().float(), other.float(), rtol=2 ** -6, atol=2 ** -6)
