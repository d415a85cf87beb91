"""The calls of a serving step together: maps, the norm, rotation and append of new rows, and
attention with capped, biased and windowed scores, over either cache."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2608_23658_amd.kvattn as K
from oracle import fp8
from oracle.qkv import norm_rope, rope_table
from oracle.scored import scored_attention
from tests.gpu_helpers import f64, require_gpu, say
from tests.scored_helpers import assert_scored
from tests.test_gpu_qkv_append import assert_rounded, raw

pytestmark = pytest.mark.gpu
HQ, HKV, D, BS, ROT, EPS = 8, 2, 128, 16, 64, 1e-5
# a layer that sees a window and one that sees everything
LAYERS = [dict(softcap=20.0, window=50), dict(softcap=0.0, window=0)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).cuda()


class Model:
    """Two layers' caches, weights and slopes; every slot starts as NaN."""

    def __init__(self, cache, nb):
        g = torch.Generator().manual_seed(5)
        self.fp8, self.nb = cache == "8bit", nb
        per = fp8.block_bytes(HKV, D) if self.fp8 else 2 * HKV * BS * D * 2
        self.kv = [torch.full((nb * per,), 0x7F if self.fp8 else 0xFF, dtype=torch.uint8,
                              device="cuda") for _ in LAYERS]
        self.w = [(1 + 0.2 * torch.randn(D, generator=g)).to(torch.bfloat16).cuda()
                  for _ in range(2)]
        self.table_h = rope_table(600, ROT)
        self.table = torch.from_numpy(self.table_h).cuda()
        self.slopes_h = (2.0 ** -np.arange(1, HQ + 1)).astype(np.float32)
        self.slopes = torch.from_numpy(self.slopes_h).cuda()

    def append(self, i, x, m, **kw):
        q, k, v = x.split((HQ, HKV, HKV), 1)
        return (K.qkv_append_fp8 if self.fp8 else K.qkv_append)(
            q, k, v, m.slot_mapping, self.kv[i], self.nb, positions=m.positions,
            rope_table=self.table, q_weight=self.w[0], k_weight=self.w[1], eps=EPS, **kw)

    def _kw(self, i, kw):
        return dict(num_kv_heads=HKV, slopes=None if i == 0 else self.slopes, **LAYERS[i], **kw)

    def prefill(self, i, q, table, m, **kw):
        return (K.prefill_chunk_scored_fp8 if self.fp8 else K.prefill_chunk_scored)(
            q, self.kv[i], self.nb, table, m.seq_lens, m.cu_seqlens_q, **self._kw(i, kw))

    def decode(self, i, q, table, m, **kw):
        return (K.decode_scored_fp8 if self.fp8 else K.decode_scored)(
            q, self.kv[i], self.nb, table, m.seq_lens, **self._kw(i, kw))

    def bits(self, i):
        b = self.kv[i].cpu().numpy()
        return fp8.to_bf16_layer(b, HKV, D) if self.fp8 else b.view(np.uint16)

    def expected(self, i, q, table, lens, cu):
        return scored_attention(raw(q), self.bits(i), table, lens, cu, dtype="bf16",
                                num_q_heads=HQ, num_kv_heads=HKV, head_dim=D,
                                scale=1 / math.sqrt(D), slopes=None if i == 0 else self.slopes_h,
                                **LAYERS[i])


def _rows(n, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(n, HQ + 2 * HKV, D, generator=g).to(torch.bfloat16)


@pytest.mark.parametrize("cache", ["bf16", "8bit"])
def test_requests_from_prompt_to_decode(cache):
    """Five requests under a budget of 80 tokens a step: prompts in chunks next to requests that
    decode, then all decode. Every step: the rotated rows against the oracle, what the cache
    holds of them, and attention over what it holds; padding rows are left alone."""
    prompts, nb, MB, T = [170, 5, 64, 1, 90], 60, 14, 80
    S = len(prompts)
    model, pool = Model(cache, nb), K.BlockPool(nb, 0)
    table_h = np.full((S, MB), -1, np.int32)
    table = torch.full((S, MB), -1, dtype=torch.int32, device="cuda")
    cached, m = [0] * S, K.StepMap.empty(S, T)
    held = [np.zeros((0, HKV, D)) for _ in range(S)], [np.zeros((0, HKV, D)) for _ in range(S)]
    for step in range(8):
        new = [p - c if c < p else 1 for p, c in zip(prompts, cached)]
        free = np.random.default_rng(step).permutation(pool.alloc(pool.num_free))
        lens, cu, slots, pos, used, want = fp8.step_map(cached, new, free, table_h, T)
        x = _rows(T, step)
        n, lens, cu = used[0], np.asarray(lens, np.int32), np.asarray(cu, np.int32)
        say("scored serving", cache, "step", step, "tokens", n)
        K.step_map(_i32(cached), _i32(new), _i32(free), table, max_tokens=T, out=m)
        table_h = want.astype(np.int32)
        kw = dict(table=model.table_h, positions=np.asarray(pos), eps=EPS)
        ref_q, size_q = norm_rope(f64(x[:, :HQ]), weight=f64(model.w[0]), **kw)
        ref_k, size_k = norm_rope(f64(x[:, HQ:HQ + HKV]), weight=f64(model.w[1]), **kw)
        for s in range(S):
            a, b = cu[s], cu[s + 1]
            held[0][s] = np.concatenate([held[0][s], ref_k[a:b]])
            held[1][s] = np.concatenate([held[1][s], f64(x[a:b, HQ + HKV:])])
        for i in range(len(LAYERS)):
            q = model.append(i, x.cuda(), m)
            assert_rounded(f64(q), ref_q, size_q, "bf16", f"q of step {step}")
            for s in range(S):       # every token the cache holds, old ones among them
                k, v = oracle.gather_kv(model.bits(i), "bf16", table_h[s], int(lens[s]), HKV, BS, D)
                if cache == "bf16":
                    ref = held[0][s]
                    top = np.abs(ref) * 2.0 ** -8 + 2.0 ** -18 * np.abs(ref).max(initial=0.0)
                    assert (np.abs(k - ref) <= top).all(), (step, s)
                    assert np.array_equal(v, held[1][s]), (step, s)
                else:   # a code is off by at most 2^-4 of the value, 2^-10 of the largest again
                        # whenever its block's exponent grows
                    for got, ref in ((k, held[0][s]), (v, held[1][s])):
                        assert (np.abs(got - ref) <= np.abs(ref).max(initial=0.0) * 0.1).all()
            keep = torch.full((T, HQ, D), 5.0, dtype=torch.bfloat16, device="cuda")
            got = model.prefill(i, q, table, m, max_seq_len=MB * BS, out=keep)
            assert_scored(got[:n], *model.expected(i, q[:n], table_h, lens, cu), cache,
                          LAYERS[i]["softcap"], f"layer {i}, step {step}")
            assert (got[n:] == 5.0).all()
            if (np.diff(cu) == 1).all():        # a decode step: the decode call sees the same
                got = model.decode(i, q[:n], table, m, max_seq_len=MB * BS)
                assert_scored(got, *model.expected(i, q[:n], table_h, lens, cu), cache,
                              LAYERS[i]["softcap"], f"decode, layer {i}, step {step}")
        taken = set(free[:used[1]].tolist())
        pool.free([j for j in free.tolist() if j not in taken])
        cached = lens.tolist()
    assert cached[0] > prompts[0]


@pytest.mark.parametrize("cache", ["bf16", "8bit"])
def test_captured_decode_steps(cache):
    """Maps, both layers' appends and decodes of a step in one graph, with one workspace,
    replayed with other work in between, against the same steps run eagerly."""
    say("scored serving graph", cache)
    S, MB, nb = 12, 20, 240
    r = np.random.default_rng(1)

    def state():
        return dict(model=Model(cache, nb), table=torch.full((S, MB), -1, dtype=torch.int32,
                                                             device="cuda"),
                    cached=torch.zeros(S, dtype=torch.int32, device="cuda"),
                    one=_i32(np.ones(S)), free=_i32(r0), m=K.StepMap.empty(S, S),
                    win=torch.zeros(S, dtype=torch.int32, device="cuda"),
                    at=torch.zeros(1, dtype=torch.int64, device="cuda"),
                    x=torch.zeros(S, HQ + 2 * HKV, D, dtype=torch.bfloat16, device="cuda"),
                    q=torch.zeros(S, HQ, D, dtype=torch.bfloat16, device="cuda"),
                    out=torch.zeros(2, S, HQ, D, dtype=torch.bfloat16, device="cuda"),
                    ws=K.workspace(K.decode_workspace_bytes(S, HQ, D, MB * BS)))

    r0 = r.permutation(nb)
    ramp = torch.arange(S, device="cuda")

    def step(x):
        x["win"].copy_(x["free"][(x["at"] + ramp).clamp(max=nb - 1)])
        K.step_map(x["cached"], x["one"], x["win"], x["table"], max_tokens=S, out=x["m"])
        for i in range(2):
            q = x["model"].append(i, x["x"], x["m"], out=x["q"])
            x["model"].decode(i, q, x["table"], x["m"], max_seq_len=MB * BS, out=x["out"][i],
                              ws=x["ws"])
        x["cached"].copy_(x["m"].seq_lens)
        x["at"].add_(x["m"].used[1:].long())

    eager, cap = state(), state()
    side = torch.cuda.Stream()
    eager["x"].copy_(_rows(S, 0)), cap["x"].copy_(_rows(S, 0))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(cap)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(cap)
    for i in range(70):
        eager["x"].copy_(_rows(S, i))
        step(eager)
        if i:
            cap["x"].copy_(_rows(S, i))
            g.replay()
        torch.cuda.synchronize()
        assert not eager["out"].isnan().any(), i
        assert torch.equal(eager["out"], cap["out"]) and torch.equal(eager["q"], cap["q"]), i
        assert torch.equal(eager["table"], cap["table"])
        for a, b in zip(eager["model"].kv, cap["model"].kv):
            assert torch.equal(a, b), i
        torch.randn(100000, device="cuda").sum().item()
    assert int(cap["at"]) == S * 5 and cap["cached"].tolist() == [70] * S


@pytest.mark.parametrize("cache", ["bf16", "8bit"])
def test_two_steps_at_once_on_their_streams(cache):
    """Two models' steps on two streams, with the tensors that the calls make, and the same
    one after the other: the same bits."""
    say("scored serving streams", cache)

    def run(streams):
        outs = []
        for n, s in enumerate(streams):
            model, T = Model(cache, 40), 200 + n
            table = torch.full((1, 40), -1, dtype=torch.int32, device="cuda")
            m, x = K.StepMap.empty(1, T), _rows(T, n).cuda()
            none, new, free = _i32([0]), _i32([T]), _i32(np.arange(40)[::-1])
            torch.cuda.synchronize()
            K.step_map(none, new, free, table, max_tokens=T, out=m, stream=s)
            q = model.append(1, x, m, stream=s)
            outs.append((model, q, model.prefill(1, q, table, m, max_seq_len=640, stream=s)))
        torch.cuda.synchronize()
        return outs

    want = run([None, None])
    got = run([torch.cuda.Stream(), torch.cuda.Stream()])
    for (a, qa, oa), (b, qb, ob) in zip(want, got):
        assert torch.equal(qa, qb) and torch.equal(a.kv[1], b.kv[1])
        assert not oa.isnan().any() and torch.equal(oa, ob)


@pytest.mark.parametrize("cache", ["bf16", "8bit"])
def test_blocks_past_4_gib(cache):
    """The same blocks at the end of a 5 GiB layer and in a small one: the same bits."""
    from tests.scored_helpers import Call
    decode = Call([1500, 40, 3000], [1, 1, 1], hq=32, hkv=8, d=128, cache=cache, softcap=20.0,
                  bias=True, window=1000, seed=9)
    chunk = Call([900, 2100], [300, 70], hq=32, hkv=8, d=128, cache=cache, softcap=20.0, bias=True,
                 window=700, seed=10)
    bias = Call([900, 2100], [300, 70], hq=32, hkv=8, d=128, cache=cache, bias=True, seed=10)
    for c, call in ((decode, Call.decode), (chunk, Call.prefill), (bias, Call.prefill)):
        want = call(c)
        per = c.kv.numel() * c.kv.element_size() // c.b.num_blocks
        nb = (5 << 30) // per
        say("scored past 4 GiB", cache, "blocks", nb)
        far = torch.full((nb * per,), 0xFF, dtype=torch.uint8, device="cuda")
        first = nb - c.b.num_blocks
        assert first * per >= 1 << 32
        far[first * per:] = c.kv.view(torch.uint8).reshape(-1)
        table = c.b.block_table
        c.b.block_table = np.where(table >= 0, table + first, table).astype(np.int32)
        c.b.num_blocks, c.kv = nb, far
        c.set_table()
        got = call(c)
        assert torch.equal(got.view(torch.int16), want.view(torch.int16)) and not got.isnan().any()
        del far, c.kv
        torch.cuda.empty_cache()


@pytest.mark.parametrize("cache", ["bf16", "8bit"])
def test_chunks_longer_than_their_context(cache):
    """Rows before a sequence's first token, and sequences without tokens, are zeros; the
    others as the oracle has them. With nothing asked for, the plain call's bits."""
    from tests.scored_helpers import Call
    c = Call([40, 100, 1], [40, 60, 1], hq=8, hkv=2, d=128, cache=cache, seed=11)
    plain = K.prefill_chunk_fp8 if cache == "8bit" else K.prefill_chunk
    for lens in ([40, 100, 1], [3, 20, 1], [0, 1, 0], [-5, 59, 1]):
        say("chunks longer than their context", cache, lens)
        c.sl.copy_(_i32(lens))
        c.b.seq_lens = np.maximum(lens, 0).astype(np.int32)
        want = plain(c.q, c.kv, c.b.num_blocks, c.bt, c.sl, c.cu, num_kv_heads=2,
                     max_seq_len=112, scale=c.scale)
        assert torch.equal(c.prefill(max_seq_len=112), want)
        for kw in (dict(bias=0.0), dict(window=7), dict(softcap=5.0), dict(softcap=5.0, window=7)):
            c.mods = dict(softcap=kw.get("softcap", 0.0), window=kw.get("window", 0))
            c.slopes = np.zeros(8, np.float32) if "bias" in kw else None
            c.dev_slopes = torch.zeros(8, device="cuda") if "bias" in kw else None
            got = c.prefill(max_seq_len=112)
            c.check(got, False, f"lens {lens} {kw}")
            for s, n in enumerate((40, 60, 1)):
                gone, first = n - max(lens[s], 0), int(c.b.cu_seqlens_q[s])
                assert gone <= 0 or not got[first:first + gone].any(), (lens, s)
        c.mods, c.slopes, c.dev_slopes = dict(softcap=0.0, window=0), None, None


@pytest.mark.parametrize("cache", ["bf16", "8bit"])
def test_empty_calls(cache):
    model = Model(cache, 4)
    before = model.kv[0].clone()
    m, table = K.StepMap.empty(0, 0), _i32(np.zeros((0, 4)))
    q = model.append(0, _rows(0, 0).cuda(), m)
    assert q.shape == (0, HQ, D)
    assert model.decode(0, q, table, m, max_seq_len=64).shape == (0, HQ, D)
    assert model.prefill(0, q, table, m, max_seq_len=64).shape == (0, HQ, D)
    torch.cuda.synchronize()
    assert torch.equal(before, model.kv[0])
