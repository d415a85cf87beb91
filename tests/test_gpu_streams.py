"""Calls on a stream of the caller's choice while the current stream is not done with
memory that it has given back, or with what a call gave it."""
import pytest
import torch

import paper_2608_23658_amd.kvattn as K
from tests.fp8_helpers import Dev8, fp8_batch
from tests.gpu_helpers import Dev, require_gpu, say
from workloads import make_batch_from_lens

pytestmark = pytest.mark.gpu
HQ, HKV, D = 8, 2, 128


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _decode_fp8():
    b, raw = fp8_batch([3000, 900, 1500, 1], [1] * 4, hq=HQ, hkv=HKV, d=D, seed=51)
    x = Dev8(b, raw)
    return lambda **kw: [x.decode(**kw)], [K.decode_workspace_bytes(4, HQ, D, 3000)]


def _prefill_chunk_fp8():
    b, raw = fp8_batch([700, 300], [200, 300], hq=HQ, hkv=HKV, d=D, seed=52)
    x = Dev8(b, raw)
    return lambda **kw: [x.prefill(**kw)], [K.prefill_workspace_bytes(2, 500, HQ, D)]


def _step_map():
    cached, new = (torch.tensor(v, dtype=torch.int32, device="cuda")
                   for v in ([30, 0, 5], [1, 900, 70]))
    free = torch.arange(64, dtype=torch.int32, device="cuda")
    table = torch.full((3, 64), 7, dtype=torch.int32, device="cuda")
    return lambda **kw: list(K.step_map(cached, new, free, table, max_tokens=1000, **kw)), []


def _bf16(decode):
    b = make_batch_from_lens([3000, 900, 1500, 1] if decode else [700, 300],
                             [1] * 4 if decode else [200, 300], dtype="bf16", num_q_heads=HQ,
                             num_kv_heads=HKV, head_dim=D, block_size=16, seed=53)
    x = Dev(b)
    ws = (K.decode_workspace_bytes(4, HQ, D, 3000) if decode else
          K.prefill_workspace_bytes(2, 500, HQ, D))
    return lambda **kw: [(x.decode if decode else x.prefill)(**kw)], [ws]


CALLS = {"decode": lambda: _bf16(True), "prefill_chunk": lambda: _bf16(False),
         "decode_fp8": _decode_fp8, "prefill_chunk_fp8": _prefill_chunk_fp8,
         "step_map": _step_map}


class Busy:
    """Some milliseconds of the current stream's time."""

    def __init__(self):
        self.x = torch.empty(1 << 31, dtype=torch.uint8, device="cuda")

    def __call__(self):
        for i in range(16):
            self.x.fill_(i)


def _bytes(t):
    return t.untyped_storage().nbytes()


@pytest.mark.parametrize("name", sorted(CALLS))
def test_memory_the_current_stream_still_writes(name):
    call, extra = CALLS[name]()
    want, busy, s = call(), Busy(), torch.cuda.Stream()
    sizes = [_bytes(t) for t in want] + extra
    want = [t.clone() for t in want]
    torch.cuda.synchronize()
    say("stream of the call", name)
    for _ in range(3):
        busy()
        for n in sizes:      # written after all that, and given back at once
            torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        got = call(stream=s)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        del got, a


@pytest.mark.parametrize("name", sorted(CALLS))
def test_results_the_current_stream_still_reads(name):
    call, _ = CALLS[name]()
    want, busy, s = [t.clone() for t in call()], Busy(), torch.cuda.Stream()
    torch.cuda.synchronize()
    say("stream of the call, results dropped", name)
    for _ in range(3):
        got = call(stream=s)
        sizes = [_bytes(t) for t in got]
        torch.cuda.current_stream().wait_stream(s)
        busy()
        kept = [t.clone() for t in got]     # after all that
        del got
        with torch.cuda.stream(s):
            junk = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes]
        torch.cuda.synchronize()
        for a, b in zip(kept, want):
            assert torch.equal(a, b)
        del junk, kept


@pytest.mark.parametrize("how", ["stream", "handle", "joined"])
@pytest.mark.parametrize("name", ["decode_fp8", "prefill_chunk_fp8", "decode", "prefill_chunk"])
def test_captured_with_a_stream_named(name, how):
    """Tensors made within a capture, for the capturing stream by name or by handle, or for
    another that joins it: the graph's own, whatever is made and dropped between replays."""
    call, sizes = CALLS[name]()
    want = [t.clone() for t in call()]
    sizes = sizes + [_bytes(t) for t in want]
    main, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    say("captured", name, how)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=main):
        if how == "joined":
            other.wait_stream(main)
            got = call(stream=other)
            main.wait_stream(other)
        else:
            got = call(stream=main if how == "stream" else main.cuda_stream)
    for _ in range(4):
        for t in got:
            t.fill_(3)
        torch.cuda.synchronize()
        g.replay()
        junk = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        del junk
