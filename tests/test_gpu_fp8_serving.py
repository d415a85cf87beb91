"""The calls of a serving step together: maps, append, prefill and decode over a cache in
8 bits, with the block pool, the elastic pool, graphs and streams they are used with."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2608_23658_amd.kvattn as K
from oracle import fp8
from tests.fp8_helpers import Dev8, assert_close, fp8_batch, u16
from tests.gpu_helpers import require_gpu, say

pytestmark = pytest.mark.gpu
HQ, HKV, D, BS = 8, 2, 128, 16
BB = fp8.block_bytes(HKV, D)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).cuda()


def _rows(n, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(n, HQ, D, generator=g).to(torch.bfloat16)
    k, v = ((torch.randn(n, HKV, D, generator=g) * size).to(torch.bfloat16) for _ in range(2))
    return q, k, v


def _oracle(raw, q, table, lens, cu):
    bits = fp8.to_bf16_layer(raw, HKV, D)
    kw = dict(dtype="bf16", num_q_heads=HQ, num_kv_heads=HKV, head_dim=D, block_size=BS,
              scale=1 / math.sqrt(D))
    ref = oracle.paged_attention(u16(q), bits, table, lens, cu, **kw)
    lay = bits.reshape(-1, 2, HKV, BS * D).copy()
    lay[:, 1] &= 0x7FFF
    return ref, oracle.paged_attention(u16(q), lay.reshape(-1), table, lens, cu, **kw)


def test_requests_from_prompt_to_decode():
    """Six requests under a budget of 96 tokens a step: prompts in chunks next to requests that
    decode, then all decode; ids come from the block pool. Every step's outputs and
    the layer's bytes against the oracle."""
    prompts, nb, MB, T = [150, 7, 64, 1, 33, 90], 64, 16, 96
    S = len(prompts)
    pool = K.BlockPool(nb, 0)
    raw = np.random.default_rng(0).integers(0, 256, nb * BB, dtype=np.uint8)
    layer = torch.from_numpy(raw.copy()).cuda()
    table_h, table = np.full((S, MB), -1, np.int32), torch.full((S, MB), -1, dtype=torch.int32,
                                                                device="cuda")
    cached, out = [0] * S, K.StepMap.empty(S, T)
    for step in range(12):
        new = [p - c if c < p else 1 for p, c in zip(prompts, cached)]
        free_h = np.random.default_rng(step).permutation(pool.alloc(pool.num_free))
        lens, cu, slots, pos, used, want = fp8.step_map(cached, new, free_h, table_h, T)
        q, k, v = _rows(T, step, size=2.0 ** (step % 5))
        say("serving step", step, "tokens", used[0], "ids", used[1])
        K.step_map(_i32(cached), _i32(new), _i32(free_h), table, max_tokens=T, out=out)
        K.kv_append_fp8(k.cuda(), v.cuda(), out.slot_mapping, layer, nb)
        keep = torch.full((T, HQ, D), 5.0, dtype=torch.bfloat16, device="cuda")
        got = K.prefill_chunk_fp8(q.cuda(), layer, nb, table, out.seq_lens, out.cu_seqlens_q,
                                  num_kv_heads=HKV, max_seq_len=MB * BS, out=keep)
        raw = fp8.append(raw, k.double().numpy(), v.double().numpy(), slots, num_kv_heads=HKV,
                         head_dim=D)
        table_h = want.astype(np.int32)
        assert out.used.tolist() == used and np.array_equal(table.cpu().numpy(), table_h)
        n = used[0]
        lens, cu = np.asarray(lens, np.int32), np.asarray(cu, np.int32)
        assert_close(got[:n], *_oracle(raw, q[:n], table_h, lens, cu), f"step {step}")
        assert (got[n:] == 5.0).all()
        a, b = (np.array(x).reshape(nb, -1)[:, :2 * HKV * BS * D + 2 * HKV]
                for x in (layer.cpu().numpy(), raw))
        a[(a & 127) == 127] = b[(b & 127) == 127] = 127
        assert np.array_equal(a, b)
        if (np.diff(cu) == 1).all():        # a decode step: the decode call sees the same
            dec = K.decode_fp8(q[:n].cuda(), layer, nb, table, out.seq_lens, num_kv_heads=HKV,
                               max_seq_len=MB * BS)
            assert_close(dec, *_oracle(raw, q[:n], table_h, lens, cu), f"decode {step}")
        taken = set(free_h[:used[1]].tolist())
        pool.free([i for i in free_h.tolist() if i not in taken])
        cached = lens.tolist()
    assert cached[0] > prompts[0]


def test_captured_decode_steps():
    """Maps, append and decode of a step in one graph, replayed with the program's own work in
    between, against the same steps run eagerly on a copy."""
    say("serving graph")
    S, MB, nb = 20, 12, 260
    r = np.random.default_rng(1)
    start = r.integers(1, 100, S)
    b, raw = fp8_batch(start.tolist(), [1] * S, hq=HQ, hkv=HKV, d=D, seed=3)
    held = [-(-int(n) // 16) for n in start]
    perm = r.permutation(nb)
    layer0 = torch.full((nb, BB), 0x7F, dtype=torch.uint8)
    tab = np.full((S, MB), -1)
    at = 0
    for s in range(S):
        for j in range(held[s]):
            tab[s, j] = perm[at]
            layer0[perm[at]] = torch.from_numpy(raw.reshape(-1, BB)[b.block_table[s, j]])
            at += 1
    free = _i32(perm[at:])

    def state():
        return dict(layer=layer0.cuda(), table=_i32(tab), cached=_i32(start),
                    at=torch.zeros(1, dtype=torch.int64, device="cuda"),
                    win=torch.zeros(S, dtype=torch.int32, device="cuda"), one=_i32(np.ones(S)),
                    m=K.StepMap.empty(S, S), out=torch.empty(S, HQ, D, dtype=torch.bfloat16,
                                                             device="cuda"),
                    q=torch.empty(S, HQ, D, dtype=torch.bfloat16, device="cuda"),
                    k=torch.empty(S, HKV, D, dtype=torch.bfloat16, device="cuda"),
                    v=torch.empty(S, HKV, D, dtype=torch.bfloat16, device="cuda"),
                    ws=K.workspace(K.decode_workspace_bytes(S, HQ, D, MB * BS)))

    ramp = torch.arange(S, device="cuda")

    def step(x):
        x["win"].copy_(free[(x["at"] + ramp).clamp(max=free.numel() - 1)])
        K.step_map(x["cached"], x["one"], x["win"], x["table"], max_tokens=S, out=x["m"])
        K.kv_append_fp8(x["k"], x["v"], x["m"].slot_mapping, x["layer"], nb)
        K.decode_fp8(x["q"], x["layer"], nb, x["table"], x["m"].seq_lens, num_kv_heads=HKV,
                     max_seq_len=MB * BS, out=x["out"], ws=x["ws"])
        x["cached"].copy_(x["m"].seq_lens)
        x["at"].add_(x["m"].used[1:].long())

    def feed(x, i):
        q, k, v = _rows(S, 100 + i, size=2.0 ** (i % 7))
        x["q"].copy_(q), x["k"].copy_(k), x["v"].copy_(v)

    eager, cap = state(), state()
    side = torch.cuda.Stream()
    feed(cap, 0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cap)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(cap)
    for i in range(40):
        feed(eager, i)
        step(eager)
        if i:
            feed(cap, i)
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager["out"], cap["out"]), i
        assert torch.equal(eager["layer"], cap["layer"]) and torch.equal(eager["table"], cap["table"])
        torch.randn(100000, device="cuda").sum().item()
    assert int(cap["at"]) > 0


@pytest.mark.parametrize("decode", [True, False])
def test_captured_with_shrinking_and_growing_lengths(decode):
    """A graph captured for its longest call, replayed at other lengths."""
    say("fp8 graph at other lengths", decode)
    full = [1100, 2000, 700] if decode else [300, 40, 900]
    new = [1, 1, 1] if decode else [100, 40, 1]
    b, raw = fp8_batch(full, new, hq=HQ, hkv=HKV, d=D, seed=31)
    dev, out = Dev8(b, raw), torch.empty(sum(new), HQ, D, dtype=torch.bfloat16, device="cuda")
    ws = K.workspace(K.decode_workspace_bytes(3, HQ, D, 2000) if decode else
                     K.prefill_workspace_bytes(3, sum(new), HQ, D))
    call = lambda **kw: (dev.decode if decode else dev.prefill)(**kw)   # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out=out, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out=out, ws=ws)
    for lens in (full, [1, 64, 700], [100, 40, 1], [0, 2, 3], full) if decode else \
            (full, [100, 40, 1], [300, 41, 65], full):
        dev.sl.copy_(_i32(lens))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        # as bits: a length past what the layer holds reaches a NaN slot, in both alike
        again = call(ws=torch.empty_like(ws))
        assert torch.equal(got.view(torch.int16), again.view(torch.int16)), lens
        torch.randn(100000, device="cuda").sum().item()


def test_streams_and_two_calls_at_once():
    """On a stream of the caller's choice, with tensors made by the call, and two calls at
    once with a workspace each: the same bits as one after the other."""
    say("fp8 streams")
    b, raw = fp8_batch([3000, 900, 1500, 1], [1, 1, 1, 1], hq=HQ, hkv=HKV, d=D, seed=41)
    p, praw = fp8_batch([700, 300], [200, 300], hq=HQ, hkv=HKV, d=D, seed=42)
    x, y = Dev8(b, raw), Dev8(p, praw)
    want_d, want_p = x.decode(), y.prefill()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        outs = [x.decode(stream=s1), y.prefill(stream=s2), x.decode(stream=s2.cuda_stream),
                y.prefill(stream=s1)]
        junk = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        for o, w in zip(outs, (want_d, want_p, want_d, want_p)):
            assert torch.equal(o, w)
        del junk


def test_elastic_pool_drained_by_copies():
    """Sequences in blocks of the elastic range of a pool: appended to, attended, then moved to
    base blocks with copy_blocks and attended again, the elastic range gone."""
    gran = K.ElasticPool.granularity()
    base_n, el_n = 96, 32
    base = -(-base_n * BB // gran) * gran
    pool = K.ElasticPool(2, base, -(-el_n * BB // gran) * gran)
    first = base // BB + 1                  # the first block wholly in the elastic range
    nb = first + el_n - 1
    say("fp8 elastic", nb, first)
    try:
        pool.commit()
        L = 200
        need = -(-L // 16)
        ids = np.arange(first, first + need)
        q, k, v = _rows(L, 7)
        t = np.arange(L)
        slots = _i32(ids[t // 16] * 16 + t % 16)
        bt, sl = _i32(ids[None]), _i32([L])
        outs = []
        for layer in range(2):
            K.kv_append_fp8(k.cuda(), v.cuda(), slots, pool.layer_ptr(layer), nb)
            outs.append(K.decode_fp8(q[:1].cuda(), pool.layer_ptr(layer), nb, bt, sl,
                                     num_kv_heads=HKV, max_seq_len=L))
        to = np.random.default_rng(1).permutation(base // BB)[:need]
        K.copy_blocks([pool.layer_ptr(0), pool.layer_ptr(1)], nb, K.fp8_block_bytes(HKV, D),
                      _i32(ids), _i32(to))
        pool.decommit()
        for layer in range(2):
            o = K.decode_fp8(q[:1].cuda(), pool.layer_ptr(layer), base // BB, _i32(to[None]), sl,
                             num_kv_heads=HKV, max_seq_len=L)
            assert torch.equal(o, outs[layer])
        torch.cuda.synchronize()
    finally:
        pool.close()


def test_blocks_past_4gib():
    """Blocks whose byte offsets need 64 bits give what the same blocks give at the start of
    a small layer."""
    nb, L, n = (1 << 32) // BB + 400, 700, 60
    say("fp8 large offsets", nb)
    big = torch.full((nb * BB,), 0x7F, dtype=torch.uint8, device="cuda")
    small = torch.full((64 * BB,), 0x7F, dtype=torch.uint8, device="cuda")
    high = (1 << 32) // BB + 1 + np.random.default_rng(2).permutation(398)[:44]
    high[3] = nb - 1
    low = np.arange(44)
    q, k, v = (x.cuda() for x in _rows(L, 3))
    t = np.arange(L)
    got = []
    for layer, blocks, ids in ((big, nb, high), (small, 64, low)):
        K.kv_append_fp8(k, v, _i32(ids[t // 16] * 16 + t % 16), layer, blocks)
        kw = dict(num_kv_heads=HKV, max_seq_len=L)
        got.append((K.decode_fp8(q[:1], layer, blocks, _i32(ids[None]), _i32([L]), **kw),
                    K.prefill_chunk_fp8(q[:n], layer, blocks, _i32(ids[None]), _i32([L]),
                                        _i32([0, n]), **kw),
                    layer.view(-1, BB)[torch.from_numpy(ids).cuda()]))
    for a, b in zip(*got):
        assert torch.equal(a, b)
