"""From the projection to the attention output, for models that the plain cache write and the
plain softmax do not serve: the calls a step makes on one layer, and the cases by which their
speed is judged.

  qkv      norms of q and k for each head, rotation by position (one axis, or time, height and
           width), and the new K and V written into their slots of the paged cache
  decode   one query token per sequence; scores capped by a tanh, biased by distance, cut to a
           window, or several of these
  prefill  the same scores for chunks of new tokens, each causal to itself and all before it

Over a cache in the rows' own type, blocks of [2 (K, V)][kv heads][16 tokens x d], a K tile in
16-byte chunks of 16 tokens each, a V tile dim by dim; or in 8 bits: e4m3 codes and, for each
kv head, K's and V's exponent byte, padded to 128 bytes. In an 8-bit K tile token r, dim j lies
at (j // 16 * 16 + r) * 16 + j % 16; in a V tile at
j // 64 * 1024 + r // 4 * 256 + j % 16 * 16 + j // 16 % 4 * 4 + r % 4.

Shapes are those of the framework's own workloads (32 query heads over 8 kv heads with head_dim
128; 64 over 8; head_dim 64).
"""
import math
import random

import torch

own = False

BS = 16                                  # tokens per block
E_MIN, E_MAX, E4M3_MAX = -117, 119, 448.0
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
SCRATCH = 256 << 20                      # one workspace for all calls of a program
EPS = 1e-6


def listed():
    return [
        # The rows of a decode step of a full batch: one token per sequence, each in a block of
        # its own, at a position of its own. Latency.
        dict(name="qkv_step", op="qkv", cache="own", dtype="bf16", hq=32, hkv=8, d=128, rot=128,
             norm=True, even=False, sections="", tokens=256, start=0, scattered=True,
             blocks=1024, max_pos=8192),
        # The rows of an 8192-token chunk that begins inside a block.
        dict(name="qkv_chunk", op="qkv", cache="own", dtype="bf16", hq=32, hkv=8, d=128, rot=128,
             norm=True, even=False, sections="", tokens=8192, start=5, scattered=False,
             blocks=640, max_pos=32768),
        # An image's tokens, with positions in time, height and width, from a program that keeps
        # its activations in fp32; adjacent dims are the pairs, half of them rotate.
        dict(name="qkv_axes_f32", op="qkv", cache="own", dtype="f32", hq=12, hkv=3, d=64, rot=32,
             norm=False, even=True, sections="4,6,6", tokens=1777, start=11, scattered=False,
             blocks=160, max_pos=4096),
        # A chunk into the cache in 8 bits.
        dict(name="qkv_chunk_8bit", op="qkv", cache="8bit", dtype="bf16", hq=64, hkv=8, d=128,
             rot=128, norm=True, even=False, sections="", tokens=4096, start=0, scattered=False,
             blocks=320, max_pos=32768),
        # One user's decode step with capped scores: the smallest attention call.
        dict(name="decode_cap_single", op="decode", cache="own", dtype="bf16", hq=32, hkv=8, d=128,
             cap=50.0, bias=False, window=0, batch=1, lo=3971, hi=3971, len_seed=3),
        # A few users with ragged contexts down to one token, bias by distance, head_dim 64.
        dict(name="decode_bias_few", op="decode", cache="own", dtype="bf16", hq=64, hkv=8, d=64,
             cap=0.0, bias=True, window=0, batch=12, lo=1, hi=4096, len_seed=4),
        # A full batch through a layer that sees the last 1024 tokens, scores capped.
        dict(name="decode_window_cap", op="decode", cache="own", dtype="bf16", hq=32, hkv=8, d=128,
             cap=50.0, bias=False, window=1024, batch=256, lo=512, hi=4096, len_seed=5),
        # Two long documents next to short sessions, over the cache in 8 bits.
        dict(name="decode_cap_long_8bit", op="decode", cache="8bit", dtype="bf16", hq=32, hkv=8,
             d=128, cap=30.0, bias=False, window=0, batch=6, lo=700, hi=131071, len_seed=6),
        # A follow-up question with bias by distance: a short chunk over a conversation.
        dict(name="prefill_bias_short", op="prefill", cache="own", dtype="bf16", hq=32, hkv=8,
             d=128, cap=0.0, bias=True, window=0, prompts=1, new_lo=201, new_hi=201, ctx_lo=6150,
             ctx_hi=6150, rows=0, lo=1, hi=1, len_seed=7),
        # A unified step over the cache in 8 bits: a chunk of a prompt and a batch of decode
        # sequences through a windowed, capped layer.
        dict(name="mixed_window_cap_8bit", op="prefill", cache="8bit", dtype="bf16", hq=32, hkv=8,
             d=128, cap=30.0, bias=False, window=2048, prompts=1, new_lo=2048, new_hi=2048,
             ctx_lo=6144, ctx_hi=6144, rows=64, lo=1024, hi=8192, len_seed=8),
        # The last 8192 tokens of a 32768-token prompt through a windowed layer.
        dict(name="prefill_window", op="prefill", cache="own", dtype="bf16", hq=32, hkv=8, d=128,
             cap=0.0, bias=False, window=4096, prompts=1, new_lo=8192, new_hi=8192, ctx_lo=24576,
             ctx_hi=24576, rows=0, lo=1, hi=1, len_seed=9),
        # A long chunk through a layer that sees all before it, scores capped.
        dict(name="prefill_cap", op="prefill", cache="own", dtype="bf16", hq=32, hkv=8, d=128,
             cap=50.0, bias=False, window=0, prompts=1, new_lo=4096, new_hi=4096, ctx_lo=12288,
             ctx_hi=12288, rows=0, lo=1, hi=1, len_seed=10),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["qkv", "qkv", "decode", "decode", "prefill", "prefill"])
    seed = rng.randrange(1 << 30)
    if op == "qkv":
        cache = rng.choice(["own", "own", "8bit"])
        dtype, hq, hkv, d = rng.choice([("bf16", 32, 8, 128), ("bf16", 64, 8, 128),
                                        ("bf16", 12, 3, 128), ("bf16", 8, 2, 64),
                                        ("f32", 8, 4, 64), ("f32", 32, 8, 128)])
        rot = rng.choice([d, d, d // 2])
        axes = rng.choice([1, 1, 3])
        first = rng.randrange(1, rot // 4)
        sections = "%d,%d,%d" % (first, rot // 4, rot // 4 - first) if axes == 3 else ""
        scattered = rng.random() < 0.5
        tokens = _log(rng, 1, 1024 if scattered else 8192 if dtype == "bf16" else 4096)
        start = 0 if scattered else rng.choice([0, rng.randrange(BS)])
        blocks = tokens * 4 if scattered else (tokens + start) // BS + 65
        return dict(op="qkv", cache=cache, dtype=dtype, hq=hq, hkv=hkv, d=d, rot=rot,
                    norm=rng.random() < 0.6, even=rng.random() < 0.4, sections=sections,
                    tokens=tokens, start=start, scattered=scattered, blocks=blocks,
                    max_pos=_log(rng, 256, 65536) + tokens)
    cap = rng.choice([0.0, 30.0, 50.0])
    bias = rng.random() < 0.35
    window = rng.choice([0, _log(rng, 16, 8192)]) if cap or bias else _log(rng, 16, 8192)
    cache = rng.choice(["own", "own", "8bit"])
    if op == "decode":
        hq, hkv, d = rng.choice([(32, 8, 128), (64, 8, 128), (16, 8, 128), (8, 8, 128),
                                 (12, 3, 128), (64, 8, 64), (8, 2, 64)])
        dtype = rng.choice(["bf16", "f32"]) if d == 64 and cache == "own" else "bf16"
        batch = _log(rng, 1, 256)
        hi = _log(rng, 64, min(131071, max(4096, 600000 // batch)))
        lo = rng.choice([1, max(1, hi // 8), hi])
        return dict(op="decode", cache=cache, dtype=dtype, hq=hq, hkv=hkv, d=d, cap=cap,
                    bias=bias, window=window, batch=batch, lo=lo, hi=hi, len_seed=seed)
    hq, hkv = rng.choice([(32, 8), (32, 8), (64, 8), (16, 8), (8, 8), (12, 3)])
    prompts = rng.choice([1, 1, 1, 2, 4, 9])
    new_hi = _log(rng, 16, 4096 // prompts)
    ctx_hi = rng.choice([0, _log(rng, 16, 8192)])
    hi = _log(rng, 64, 8192)
    return dict(op="prefill", cache=cache, dtype="bf16", hq=hq, hkv=hkv, d=128, cap=cap, bias=bias,
                window=window, prompts=prompts, new_lo=rng.choice([new_hi, max(1, new_hi // 6)]),
                new_hi=new_hi, ctx_lo=ctx_hi // 2, ctx_hi=ctx_hi,
                rows=rng.choice([0, 0, _log(rng, 1, 64)]), lo=max(1, hi // 8), hi=hi,
                len_seed=seed)


# ---------------------------------------------------------------------------
# Lengths: fixed by the case, so that every seed does the same work.

def _lens(c):
    """(context lengths including the new tokens, new tokens), prompts first."""
    r = random.Random(c["len_seed"])
    if c["op"] == "prefill":
        new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(c["prompts"])]
        lens = [n + r.randint(c["ctx_lo"], c["ctx_hi"]) for n in new]
        lens += [r.randint(c["lo"], c["hi"]) for _ in range(c["rows"])]
        return lens, new + [1] * c["rows"]
    lens = [r.randint(c["lo"], c["hi"]) for _ in range(c["batch"])]
    if c["lo"] < c["hi"] and c["hi"] > 65536:      # two long ones, the rest short sessions
        lens = ([c["hi"], c["hi"] // 2] + [r.randint(c["lo"], 4096 + c["lo"])
                                           for _ in range(c["batch"] - 2)])[:c["batch"]]
    return lens, [1] * len(lens)


# ---------------------------------------------------------------------------
# The layouts

def _block_bytes(hkv, d):
    return 2 * hkv * BS * d + -(-2 * hkv // 128) * 128


def _codes(layer, hkv, d):
    """An 8-bit layer's K and V codes as views [blocks, 2, hkv, tile]."""
    return layer[:, :2 * hkv * BS * d].unflatten(1, (2, hkv, BS * d)).view(torch.float8_e4m3fn)


def _exps(layer, hkv, d):
    """An 8-bit layer's exponent bytes as a view [blocks, hkv, 2 (K, V)]."""
    at = 2 * hkv * BS * d
    return layer[:, at:at + 2 * hkv].unflatten(1, (hkv, 2))


def _places(cache, dtype, d, dev):
    """Where token r, dim j lies in a K tile and in a V tile, [2, 16, d]."""
    r, j = torch.arange(BS, device=dev)[:, None], torch.arange(d, device=dev)[None, :]
    if cache == "8bit":
        return torch.stack([(j // 16 * 16 + r) * 16 + j % 16,
                            j // 64 * 1024 + r // 4 * 256 + j % 16 * 16 + j // 16 % 4 * 4 + r % 4])
    vec = 16 // TORCH[dtype].itemsize
    return torch.stack([(j // vec * BS + r) * vec + j % vec, j * BS + r])


def _pow2(e):
    return ((e + 127) << 23).view(torch.float32)


def _exponent(amax):
    """The least e with amax <= 448 * 2 ** e, within the exponents in use."""
    return (((amax.view(torch.int32) + 0x1fffff) >> 23) - 135).clamp(E_MIN, E_MAX)


# ---------------------------------------------------------------------------
# Inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _layer(c, num_blocks, g):
    """A layer whose blocks hold numbers of each head's own size, those past a sequence's end
    too, as a used pool does."""
    hkv, d = c["hkv"], c["d"]
    head = 2.0 ** torch.linspace(-1, 1, hkv, device="cuda")[:, None]
    if c["cache"] == "8bit":
        layer = torch.zeros(num_blocks, _block_bytes(hkv, d), dtype=torch.uint8, device="cuda")
    else:
        layer = torch.empty(num_blocks, 2, hkv, BS * d, dtype=TORCH[c["dtype"]], device="cuda")
    step = max(1, (1 << 27) // (2 * hkv * BS * d))
    for b in range(0, num_blocks, step):
        n = min(step, num_blocks - b)
        x = torch.randn(n, 2, hkv, BS * d, generator=g, device="cuda")
        x[:, 1] *= head
        if c["cache"] == "8bit":
            e = _exponent(x.abs().amax(-1))
            _exps(layer, hkv, d)[b:b + n] = (e + 127).to(torch.uint8).transpose(1, 2)
            _codes(layer, hkv, d)[b:b + n] = (x * _pow2(-e)[..., None]).to(torch.float8_e4m3fn)
        else:
            layer[b:b + n] = x.to(layer.dtype)
    return layer


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _rope_table(length, rot):
    """cos then sin of the rot / 2 pairs' angles, one row per position, from 64 bits."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    a = torch.arange(length, device="cuda", dtype=torch.float64)[:, None] * f[None, :]
    return torch.cat([a.cos(), a.sin()], 1).float()


def _sections(c):
    return tuple(int(x) for x in c["sections"].split(",")) if c["sections"] else (c["rot"] // 2,)


def _prepare_qkv(c, g):
    T, hq, hkv, d, nb = c["tokens"], c["hq"], c["hkv"], c["d"], c["blocks"]
    dt = TORCH[c["dtype"]]
    perm = torch.randperm(nb, generator=g, device="cuda")
    t = torch.arange(c["start"], c["start"] + T, device="cuda")
    if c["scattered"]:
        slots = perm[:T] * BS + torch.randint(0, BS, (T,), generator=g, device="cuda")
        pos = torch.randint(0, c["max_pos"], (T,), generator=g, device="cuda")
    else:
        slots, pos = perm[t // BS] * BS + t % BS, t - t[0] + c["max_pos"] - T
    sections = _sections(c)
    if len(sections) > 1:                # a picture 40 tokens wide at one point in time
        i = torch.arange(T, device="cuda")
        pos = torch.stack([pos[:1].expand(T), i // 40 % c["max_pos"], i % 40])
    else:
        pos = pos[None]
    # heads of different sizes, as a projection gives them
    heads = hq + 2 * hkv
    size = 2.0 ** torch.randint(-1, 3, (1, heads, 1), generator=g, device="cuda")
    rows = torch.randn(T, heads, d, generator=g, device="cuda").mul_(size)
    w = [(1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dt) if c["norm"] else None
         for _ in range(2)]
    return dict(c=c, rows=rows.to(dt).view(T, heads * d), slots=slots.to(torch.int32),
                pos=pos.to(torch.int32).contiguous(), table=_rope_table(c["max_pos"], c["rot"]),
                q_weight=w[0], k_weight=w[1], layer=_layer(c, nb, g), num_blocks=nb,
                sections=sections)


def prepare(case, seed):
    g = _gen(seed)
    c = case
    if c["op"] == "qkv":
        return _prepare_qkv(c, g)
    lens, new = _lens(c)
    need = [-(-n // BS) for n in lens]
    nb = -(-(sum(need) * 11) // 10 // 32) * 32 + 32
    layer = _layer(c, nb, g)
    perm = torch.randperm(nb, generator=g, device="cuda").to(torch.int32)
    at = torch.tensor([0] + need, device="cuda").cumsum(0)
    col = torch.arange(max(need), device="cuda")[None, :]
    table = torch.where(col < (at[1:] - at[:-1])[:, None],
                        perm[(at[:-1, None] + col).clamp(max=nb - 1)], -1)
    # queries of a few times unit size: scores reach where a cap bends them
    q = 3 * torch.randn(sum(new), c["hq"], c["d"], generator=g, device="cuda")
    slopes = None
    if c["bias"]:                        # a geometric series over the heads
        slopes = 2.0 ** (-8.0 * torch.arange(1, c["hq"] + 1, device="cuda") / c["hq"])
    return dict(c=c, q=q.to(TORCH[c["dtype"]]), layer=layer, table=table.contiguous(),
                num_blocks=nb, lens=_i32(lens), max_len=max(lens), slopes=slopes,
                cu=torch.cat([_i32([0]), _i32(new).cumsum(0).to(torch.int32)]),
                chunks=list(zip(lens, new)),      # the scheduler's own copy
                ws=torch.empty(SCRATCH, dtype=torch.uint8, device="cuda"))


# ---------------------------------------------------------------------------
# A pass

def run(s):
    if own:
        return _run_own(s)
    if s["c"]["op"] == "qkv":
        return _plain_qkv(s)
    if s["c"]["op"] == "decode":
        return _plain_rows(s, s["q"], s["table"], s["lens"])
    return _plain_prefill(s)


def _run_own(s):
    import paper_2608_23658_amd.kvattn as K
    c = s["c"]
    wide = c["cache"] == "own"
    if c["op"] == "qkv":
        hq, hkv, d = c["hq"], c["hkv"], c["d"]
        q, k, v = s["rows"].view(-1, hq + 2 * hkv, d).split_with_sizes((hq, hkv, hkv), 1)
        call = K.qkv_append if wide else K.qkv_append_fp8
        q = call(q, k, v, s["slots"], s["layer"], s["num_blocks"], positions=s["pos"],
                 rope_table=s["table"], sections=s["sections"], interleaved=c["even"],
                 q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS)
        return _rows_and_cache(s, q)
    if c["op"] == "decode":
        call = K.decode_scored if wide else K.decode_scored_fp8
        return call(s["q"], s["layer"], s["num_blocks"], s["table"], s["lens"],
                    num_kv_heads=c["hkv"], max_seq_len=s["max_len"], softcap=c["cap"],
                    slopes=s["slopes"], window=c["window"], ws=s["ws"])
    call = K.prefill_chunk_scored if wide else K.prefill_chunk_scored_fp8
    return call(s["q"], s["layer"], s["num_blocks"], s["table"], s["lens"], s["cu"],
                num_kv_heads=c["hkv"], max_seq_len=s["max_len"], softcap=c["cap"],
                slopes=s["slopes"], window=c["window"], ws=s["ws"])


def _rows_and_cache(s, q):
    """The queries, and the cache as it stands: 8 bits as the codes' and exponents' numbers."""
    c = s["c"]
    if c["cache"] == "own":
        return dict(q=q, layer=s["layer"])
    return dict(q=q, codes=_codes(s["layer"], c["hkv"], c["d"]),
                scales=_exps(s["layer"], c["hkv"], c["d"]).view(torch.float8_e8m0fnu))


def _plain_rotate(x, s):
    """x [T, heads, d] in 32 bits by the table's rows of its positions."""
    c, rot = s["c"], s["c"]["rot"]
    axis = torch.repeat_interleave(torch.arange(len(s["sections"]), device=x.device),
                                   torch.tensor(s["sections"], device=x.device),
                                   output_size=rot // 2)
    pair = torch.arange(rot // 2, device=x.device)
    at = s["pos"].long()[axis]                                           # [rot / 2, T]
    cos, sin = (s["table"][at, (pair + i * (rot // 2))[:, None]].t()[:, None, :] for i in range(2))
    if c["even"]:
        a, b = x[..., :rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1 if c["even"] else -2).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_norm(x, w):
    if w is None:
        return x
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()


def _plain_qkv(s):
    c, layer = s["c"], s["layer"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    x = s["rows"].view(-1, hq + 2 * hkv, d).float()
    q = _plain_rotate(_plain_norm(x[:, :hq], s["q_weight"]), s).to(s["rows"].dtype)
    k = _plain_rotate(_plain_norm(x[:, hq:hq + hkv], s["k_weight"]), s)
    kv = torch.stack([k, x[:, hq + hkv:]], 1)                            # [T, 2, hkv, d]
    dev = x.device
    block, r = (s["slots"] // BS).long(), (s["slots"] % BS).long()
    place = _places(c["cache"], c["dtype"], d, dev)[:, r].transpose(0, 1)[:, :, None, :]
    heads = torch.arange(hkv, device=dev)[None, None, :, None]
    which = torch.arange(2, device=dev)[None, :, None, None]
    if c["cache"] == "own":
        layer[block[:, None, None, None], which, heads, place] = kv.to(layer.dtype)
        return _rows_and_cache(s, q)
    # every token does its whole block's part: tokens of one block compute and store the same
    T = len(block)
    run_id = torch.cat([block.new_zeros(1), (block[1:] != block[:-1]).long().cumsum(0)])
    codes, exps = _codes(layer, hkv, d).view(torch.uint8), _exps(layer, hkv, d)
    fresh = torch.zeros(T, device=dev).index_reduce_(0, run_id, (r == 0).float(), "amax")
    fresh = fresh[run_id][:, None, None] > 0
    amax = torch.zeros(T, 2, hkv, device=dev).index_reduce_(0, run_id, kv.abs().amax(-1), "amax")
    e_new = _exponent(amax[run_id])
    e_old = exps[block].transpose(1, 2).int() - 127
    e = torch.where(fresh, e_new, torch.maximum(e_old, e_new))
    grown = torch.where(fresh, 0, e - e_old)
    tile = codes[block]                                                  # [T, 2, hkv, BS * d]
    scaled = tile.view(torch.float8_e4m3fn).float() * _pow2(-grown)[..., None]
    codes[block] = torch.where(grown[..., None] > 0,
                               scaled.to(torch.float8_e4m3fn).view(torch.uint8), tile)
    new = (kv * _pow2(-e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    codes[block[:, None, None, None], which, heads, place] = new
    exps[block] = (e + 127).to(torch.uint8).transpose(1, 2)
    return _rows_and_cache(s, q)


def _plain_context(s, ids):
    """K and V [..., hkv, tokens, d] in 32 bits of blocks ids [..., blocks]."""
    c, layer, hkv, d = s["c"], s["layer"], s["c"]["hkv"], s["c"]["d"]
    ids = ids.clamp(min=0).long()
    place = _places(c["cache"], c["dtype"], d, layer.device).flatten(1)
    if c["cache"] == "own":
        tiles = layer[ids].float()                                       # [..., n, 2, hkv, tile]
    else:
        tiles = _codes(layer, hkv, d).view(torch.uint8)[ids].view(torch.float8_e4m3fn).float()
        tiles *= _pow2(_exps(layer, hkv, d)[ids].int() - 127).transpose(-1, -2)[..., None]
    return [tiles[..., i, :, :][..., place[i]].unflatten(-1, (BS, d)).transpose(-4, -3)
            .flatten(-3, -2) for i in range(2)]


def _plain_attend(s, q, k, v, ago):
    """q [..., hkv, G, n, d], k and v [..., hkv, tokens, d]; ago [..., n, tokens]: how far a key
    lies behind a row's own token, below zero for those that come after it."""
    c = s["c"]
    sc = torch.matmul(q.flatten(-3, -2), k.transpose(-2, -1).contiguous())
    sc = sc.unflatten(-2, q.shape[-3:-1]).mul_(1 / math.sqrt(c["d"]))
    if c["cap"]:
        sc.div_(c["cap"]).tanh_().mul_(c["cap"])
    ago = ago[..., None, None, :, :]
    if c["bias"]:
        sc.sub_(s["slopes"].view(c["hkv"], -1)[..., None, None] * ago)
    seen = (ago >= 0) & (ago < c["window"]) if c["window"] else ago >= 0
    sc.masked_fill_(~seen, -math.inf)
    sc = sc.sub_(sc.amax(-1, keepdim=True)).exp_()
    den = sc.sum(-1, keepdim=True)
    return torch.matmul(sc.flatten(-3, -2), v).unflatten(-2, q.shape[-3:-1]).div_(den)


def _plain_rows(s, q, table, lens):
    """One row per sequence, its last token: q [B, hq, d]."""
    k, v = _plain_context(s, table)
    ago = lens[:, None] - 1 - torch.arange(k.shape[-2], device=q.device)[None, :]
    v = v.masked_fill_((ago < 0)[:, None, :, None], 0)
    rows = q.float().unflatten(1, (s["c"]["hkv"], -1))[..., None, :]
    return _plain_attend(s, rows, k, v, ago[:, None, :]).squeeze(-2).flatten(1, 2).to(q.dtype)


def _plain_chunk(s, q, ids, L):
    """The last rows of one sequence: q [n, hq, d]; a window's rows see no block before first."""
    n, w = len(q), s["c"]["window"]
    first = max(0, L - n - w + 1) // BS if w else 0
    k, v = (x[:, :L - first * BS] for x in _plain_context(s, ids[first:-(-L // BS)]))
    rows = q.float().unflatten(1, (s["c"]["hkv"], -1)).permute(1, 2, 0, 3)      # [hkv, G, n, d]
    own_pos = L - n + torch.arange(n, device=q.device)
    ago = own_pos[:, None] - (first * BS + torch.arange(k.shape[1], device=q.device))[None, :]
    out = _plain_attend(s, rows, k, v, ago)
    return out.permute(2, 0, 1, 3).flatten(1, 2).to(q.dtype)


def _plain_prefill(s):
    """Chunks of several rows one by one, the sequences that add one row together."""
    out, at, q = torch.empty_like(s["q"]), 0, s["q"]
    rows = s["c"]["rows"]                           # they come last
    several = s["chunks"][:len(s["chunks"]) - rows]
    for i, (L, n) in enumerate(several):
        out[at:at + n] = _plain_chunk(s, q[at:at + n], s["table"][i], L)
        at += n
    if rows:
        width = -(-max(L for L, _ in s["chunks"][-rows:]) // BS)
        out[at:] = _plain_rows(s, q[at:], s["table"][-rows:, :width], s["lens"][-rows:])
    return out


# ---------------------------------------------------------------------------
# What a pass cannot do without

def _work_qkv(c):
    T, row, e = c["tokens"], c["hkv"] * c["d"], TORCH[c["dtype"]].itemsize
    blocks = T if c["scattered"] else (T + c["start"] + BS - 1) // BS
    cache = 2 * T * row * (1 if c["cache"] == "8bit" else e)
    if c["cache"] == "8bit":
        cache += 4 * blocks * c["hkv"]              # exponents, read and written
    axes = len(_sections(c))
    rows = T if axes == 1 else min(T, 40 + T // 40)
    return {"bytes": (2 * c["hq"] * c["d"] + 2 * row) * T * e + cache + 4 * T * (1 + axes)
            + 4 * c["rot"] * min(rows, c["max_pos"]),
            "flops": T * (c["hq"] * c["d"] + row) * (3 * c["norm"] + 3)}


def work(case):
    c = case
    if c["op"] == "qkv":
        return _work_qkv(c)
    lens, new = _lens(c)
    w = c["window"] or max(lens)
    # rows see 1 .. of their own context, at most w; tokens: those that any row sees
    pairs, tokens, blocks = 0, 0, 0
    for L, n in zip(lens, new):
        short = min(n, max(0, w - (L - n)))         # rows that see all before them
        pairs += short * (L - n) + short * (short + 1) // 2 + (n - short) * w
        first = max(0, L - n - w + 1)
        tokens += L - first
        blocks += -(-L // BS) - first // BS
    e = 1 if c["cache"] == "8bit" else TORCH[c["dtype"]].itemsize
    kv = 2 * tokens * c["hkv"] * c["d"] * e + (2 * blocks * c["hkv"] if e == 1 else 0)
    qo = 2 * sum(new) * c["hq"] * c["d"] * TORCH[c["dtype"]].itemsize
    return {"bytes": kv + qo + 4 * blocks + 8 * len(lens) + (4 * c["hq"] if c["bias"] else 0),
            "flops": 4 * c["d"] * c["hq"] * pairs}


# ---------------------------------------------------------------------------
# The same results in 64 bits, from the definition

def _exact_kv(s, ids):
    """Tokens [hkv, 16 * blocks, d] in 64 bits of the blocks ids: K and V."""
    c, hkv, d = s["c"], s["c"]["hkv"], s["c"]["d"]
    ids, size = ids.long(), BS * d
    if c["cache"] == "own":
        vec = 16 // TORCH[c["dtype"]].itemsize
        t = s["layer"][ids].double()
        k = t[:, 0].view(-1, hkv, d // vec, BS, vec).permute(1, 0, 3, 2, 4)
        v = t[:, 1].view(-1, hkv, d, BS).permute(1, 0, 3, 2)
    else:
        raw = s["layer"][ids]
        e = raw[:, 2 * hkv * size:2 * hkv * size + 2 * hkv].view(-1, hkv, 2).double() - 127
        k, v = (raw[:, i * hkv * size:(i + 1) * hkv * size].contiguous()
                .view(torch.float8_e4m3fn).double().view(-1, hkv, size)
                * torch.exp2(e[:, :, i])[..., None] for i in range(2))
        k = k.view(-1, hkv, d // 16, BS, 16).permute(1, 0, 3, 2, 4)
        v = v.view(-1, hkv, d // 64, 4, 16, 4, 4).permute(1, 0, 3, 6, 2, 5, 4)
    return k.reshape(hkv, -1, d), v.reshape(hkv, -1, d)


def _exact_attention(s):
    c = s["c"]
    hq, hkv = c["hq"], c["hkv"]
    out, at = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), 0
    for i, (L, n) in enumerate(s["chunks"]):
        k, v = (x[:, :L] for x in _exact_kv(s, s["table"][i, :-(-L // BS)]))
        keys = torch.arange(L, device="cuda")
        step = max(1, (1 << 26) // L)
        for h in range(hq):
            kt, vh = k[h * hkv // hq].t().contiguous(), v[h * hkv // hq].contiguous()
            for r in range(0, n, step):
                x = s["q"][at + r:at + min(n, r + step), h].double() @ kt / math.sqrt(c["d"])
                if c["cap"]:
                    x = c["cap"] * torch.tanh(x / c["cap"])
                p = L - n + r + torch.arange(len(x), device="cuda")
                far = p[:, None] - keys[None, :]
                if c["bias"]:
                    x = x - float(s["slopes"][h]) * far
                gone = far < 0
                if c["window"]:
                    gone |= far >= c["window"]
                out[at + r:at + r + len(x), h] = torch.softmax(x.masked_fill(gone, -math.inf), -1) @ vh
        at += n
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_qkv(s) if case["op"] == "qkv" else _exact_attention(s)


def _exact_rows(s, x, w):
    """One head's rows [T, d] in 64 bits: normed, each pair turned as a complex number."""
    import numpy as np
    c, rot = s["c"], s["c"]["rot"]
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * w
    table, pos = s["host_table"], s["host_pos"]
    x, axes = x.copy(), np.repeat(np.arange(len(s["sections"])), s["sections"])
    for i, axis in enumerate(axes):
        a, b = (2 * i, 2 * i + 1) if c["even"] else (i, i + rot // 2)
        turn = table[pos[axis], i] + 1j * table[pos[axis], i + rot // 2]
        z = (x[:, a] + 1j * x[:, b]) * turn
        x[:, a], x[:, b] = z.real, z.imag
    return x


def _exact_qkv(s):
    """Whole rows of the cache as they should lie; codes before their rounding to e4m3."""
    import numpy as np
    c = s["c"]
    hq, hkv, d, size = c["hq"], c["hkv"], c["d"], BS * c["d"]
    s["host_table"], s["host_pos"] = s["table"].double().cpu().numpy(), s["pos"].cpu().numpy()
    rows = s["rows"].view(-1, hq + 2 * hkv, d).double().cpu().numpy()
    w = [None if x is None else x.double().cpu().numpy() for x in (s["q_weight"], s["k_weight"])]
    q = np.stack([_exact_rows(s, rows[:, h], w[0]) for h in range(hq)], 1)
    k = np.stack([_exact_rows(s, rows[:, h], w[1]) for h in range(hq, hq + hkv)], 1)
    x = np.stack([k, rows[:, hq + hkv:]], 1)                             # [T, 2, hkv, d]
    slots, j = s["slots"].cpu().numpy().astype(np.int64), np.arange(d)
    if c["cache"] == "own":
        vec = 16 // TORCH[c["dtype"]].itemsize
        layer = s["layer"].double().cpu().numpy()
        b, r = slots // BS, slots % BS
        for h in range(hkv):
            layer[b[:, None], 0, h, (j // vec * BS + r[:, None]) * vec + j % vec] = x[:, 0, h]
            layer[b[:, None], 1, h, j * BS + r[:, None]] = x[:, 1, h]
        return dict(q=q, layer=layer)
    raw = s["layer"].cpu()
    code = raw[:, :2 * hkv * size].contiguous().view(torch.float8_e4m3fn).double()
    code = code.view(-1, 2, hkv, size).numpy().copy()
    exps = raw[:, 2 * hkv * size:2 * hkv * size + 2 * hkv].view(-1, hkv, 2).numpy().astype(np.int64)
    at = 0
    while at < len(slots):
        b, end = slots[at] // BS, at
        while end < len(slots) and slots[end] // BS == b:
            end += 1
        in_block = slots[at:end] % BS
        top = np.abs(x[at:end]).max(axis=(0, 3))                         # [2, hkv]
        e = np.ceil(np.log2(np.maximum(top, 1e-300) / E4M3_MAX)).astype(np.int64)
        e -= top <= E4M3_MAX * np.exp2(e - 1.0)       # log2 may be a hair off a whole number
        e += top > E4M3_MAX * np.exp2(e * 1.0)
        e = np.clip(e, E_MIN, E_MAX)
        old = exps[b].T - 127
        if not (in_block == 0).any():
            e = np.maximum(e, old)
            code[b] *= np.exp2(np.minimum(old - e, 0) * 1.0)[..., None]
        exps[b] = e.T + 127
        for t, r in zip(range(at, end), in_block):
            y = x[t] * np.exp2(-e * 1.0)[..., None]
            code[b, 0][:, (j // 16 * 16 + r) * 16 + j % 16] = y[0]
            code[b, 1][:, j // 64 * 1024 + r // 4 * 256 + j % 16 * 16 + j // 16 % 4 * 4
                       + r % 4] = y[1]
        at = end
    return dict(q=q, codes=code, scales=np.exp2(exps - 127.0))
