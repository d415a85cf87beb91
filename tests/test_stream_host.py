"""Where the tensors that a call makes come from when it is given a stream: the
binding runs here without a GPU, on a library and streams that only note what is asked
of them."""
import contextlib

import pytest
import torch

import paper_2608_23658_amd.kvattn as K


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


HERE, OTHER = Stream(0x1000), Stream(0x2000)


class Library:
    """Every call succeeds; sizes are a page, counts 64."""

    def __getattr__(self, name):
        return lambda *a: (4096 if name.endswith("bytes") else
                           64 if name.endswith(("threads", "waves")) else K.KV_OK)


class Notes:
    def __init__(self):
        self.on, self.made, self.recorded = HERE, [], []


@pytest.fixture
def notes(monkeypatch):
    n = Notes()

    @contextlib.contextmanager
    def stream(s):
        before, n.on = n.on, s
        try:
            yield
        finally:
            n.on = before

    def noting(make):
        def made(*a, **kw):
            t = make(*a, **dict(kw, device="cpu") if "device" in kw else kw)
            n.made.append((t.data_ptr(), n.on.cuda_stream))
            return t
        return made

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: n.on)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream(0))
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch, "empty", noting(torch.empty))
    monkeypatch.setattr(torch, "empty_like", noting(torch.empty_like))
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda t, s: n.recorded.append((t.data_ptr(), s.cuda_stream)))
    for check in ("_require_cuda", "_require_here"):
        monkeypatch.setattr(K, check, lambda *ts: None)
    monkeypatch.setattr(K, "lib", Library)
    return n


def _i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def _batch():
    q = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    return q, torch.zeros(1 << 17, dtype=torch.uint8), 2, _i32(4, 3), _i32(4)


KW = dict(num_kv_heads=2, max_seq_len=48)
CALLS = {
    "decode_fp8": lambda **kw: K.decode_fp8(*_batch(), **KW, **kw),
    "prefill_chunk_fp8": lambda **kw: K.prefill_chunk_fp8(*_batch(), _i32(5), **KW, **kw),
    "decode": lambda **kw: K.decode(*_batch(), **KW, **kw),
    "decode_two_tensor": lambda **kw: K.decode_two_tensor(
        _batch()[0], _batch()[1], 1, _batch()[1], 1, *_batch()[3:], **KW, **kw),
    "prefill_chunk": lambda **kw: K.prefill_chunk(*_batch(), _i32(5), **KW, **kw),
    "probe_mfma": lambda **kw: K.probe_mfma(1, 1, **kw),
    "probe_read_blocks": lambda **kw: K.probe_read_blocks(
        *_batch()[1:], head_dim=128, dtype=torch.bfloat16, **KW, **kw),
    "step_map": lambda **kw: K.step_map(_i32(4), _i32(4), _i32(5), _i32(4, 3), max_tokens=10,
                                        **kw),
}


def _check(notes, call, stream, handle):
    got = call(stream=stream)
    got = got if isinstance(got, tuple) else (got,)
    assert notes.made and all(on == handle for _, on in notes.made), "made for another stream"
    for t in got:      # the caller's from now on, who is on the current stream
        assert (t.data_ptr(), HERE.cuda_stream) in notes.recorded
    assert notes.on is HERE


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("stream,handle", [(OTHER, 0x2000), (0x3000, 0x3000), (0, 0)])
def test_made_for_the_stream_of_the_call(notes, name, stream, handle):
    """The allocator hands memory out again as soon as the stream it was made for is done
    with it in order: made for the current stream, another stream's launch would write
    what work still pending there reads or writes."""
    _check(notes, CALLS[name], stream, handle)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_made_for_the_current_stream_without_one(notes, name):
    CALLS[name]()
    assert notes.made and all(on == HERE.cuda_stream for _, on in notes.made)
    assert not notes.recorded
