"""The step maps on the GPU against the token-by-token oracle."""
import numpy as np
import pytest
import torch

import paper_2608_23658_amd.kvattn as K
from oracle import fp8
from tests.gpu_helpers import require_gpu, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).cuda()


def _check(cached, new, free, table, max_tokens, **kw):
    t = _i32(table)
    m = K.step_map(_i32(cached), _i32(new), _i32(free), t, max_tokens=max_tokens, **kw)
    torch.cuda.synchronize()
    lens, cu, slots, pos, used, want = fp8.step_map(cached, new, free, table, max_tokens)
    assert m.cu_seqlens_q.tolist() == cu
    assert m.seq_lens.tolist() == lens
    assert m.used.tolist() == used
    assert np.array_equal(t.cpu().numpy(), want)
    assert np.array_equal(m.slot_mapping.cpu().numpy(), np.asarray(slots, np.int32))
    assert np.array_equal(m.positions.cpu().numpy(), np.asarray(pos, np.int32))
    return m


def _random(seed, S, MB, hi_new, most=None):
    r = np.random.default_rng(seed)
    cached = r.integers(0, MB * 16 + 1, S)
    new = np.where(r.random(S) < 0.5, 1, r.integers(0, hi_new + 1, S))
    ids = r.permutation(S * MB + 64)
    table = np.full((S, MB), -1)
    at = 0
    for s in range(S):
        n = -(-int(cached[s]) // 16)
        table[s, :n] = ids[at:at + n]
        at += n
    return cached, new, ids[at:] if most is None else ids[at:at + most], table


@pytest.mark.parametrize("S,MB,hi,T", [
    (1, 4, 1, 1), (1, 64, 1000, 1024), (3, 7, 40, 50), (256, 32, 1, 256), (257, 33, 90, 5000),
    (1000, 20, 17, 100), (4096, 5, 9, 20000), (4097, 5, 9, 20001), (9001, 3, 6, 30000),
    (1024, 6, 30, 9000), (1025, 6, 30, 9000), (2048, 5, 9, 9000), (2049, 5, 9, 9000),
])
def test_against_the_oracle(S, MB, hi, T):
    say("step map", S, MB, hi, T)
    _check(*_random(S + T, S, MB, hi), T)


def test_lengths_of_zero_and_nothing_new():
    say("step map: empty requests")
    table = np.full((4, 2), -1)
    _check([0, 0, 0, 0], [0, 0, 0, 0], [5], table, 3)
    _check([0, 5, 0, 16], [0, 1, 0, 1], [5, 6], [[-1, -1], [9, -1], [-1, -1], [3, -1]], 7)
    _check([0], [0], np.zeros(0), [[-1]], 0)
    m = _check(np.zeros(0), np.zeros(0), [1], np.zeros((0, 3)), 5)
    assert m.cu_seqlens_q.tolist() == [0]


def test_full_tables_budgets_and_negative_lengths():
    say("step map: no room")
    table = [[1, 2], [3, 4], [-1, -1], [5, -1]]
    _check([32, 31, -4, 16], [3, 3, 3, -7], [10, 11], table, 64)      # rows full, negatives
    _check([32, 20, 0, 16], [1, 9, 30, 5], [10, 11, 12], table, 13)   # cut inside a request
    _check([32, 20, 0, 16], [1, 9, 30, 5], [10, 11, 12], table, 9)    # cut between requests
    _check([0, 0, 0, 0], [2 ** 31 - 1] * 4, [10, 11, 12], np.full((4, 2), -1), 100)


def test_too_few_ids_and_ids_that_are_none():
    say("step map: too few ids")
    c, n, free, table = _random(8, 60, 9, 100, most=20)
    m = _check(c, n, free, table, 4000)
    assert int(m.used[1]) > 20 and (m.slot_mapping < 0).any()
    _check(c, n, np.zeros(0), table, 4000)
    _check([20], [3], [2 ** 31 - 1], [[0, -1, -1]], 4)       # the partial block is none


def test_large_ids_reach_the_last_slot():
    say("step map: large ids")
    top = (2 ** 31 - 16) // 16
    _check([0], [20], [top, 7], [[-1, -1]], 20)
    # an id whose slots pass 32 bits gives none
    t = _i32([[-1, -1]])
    m = K.step_map(_i32([0]), _i32([20]), _i32([top + 1, 7]), t, max_tokens=20)
    assert m.slot_mapping.tolist() == [-1] * 16 + [112 + i for i in range(4)]


def test_same_again_other_stream_and_kept_outputs():
    say("step map: again, stream, out")
    c, n, free, table = _random(5, 300, 12, 60)
    a = _check(c, n, free, table, 6000)
    out = K.StepMap.empty(300, 6000)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    b = _check(c, n, free, table, 6000, out=out, stream=st)
    assert b is out
    for x, y in zip(a, b):
        assert torch.equal(x, y)


def test_captured_steps_replayed():
    """A graph of one decode step: the maps, and the lengths carried over."""
    say("step map: graph")
    S, MB = 40, 8
    r = np.random.default_rng(3)
    start = r.integers(0, 20, S)
    table0 = np.full((S, MB), -1)
    for s in range(S):
        n = -(-int(start[s]) // 16)
        table0[s, :n] = 1000 + s * MB + np.arange(n)
    cached, new, table = _i32(start), _i32(np.ones(S)), _i32(table0)
    free, out = _i32(np.arange(500)), K.StepMap.empty(S, S + 3)
    cursor = torch.zeros(1, dtype=torch.int64, device="cuda")
    window = torch.zeros(S, dtype=torch.int32, device="cuda")
    ramp = torch.arange(S, device="cuda")

    def step():
        window.copy_(free[(cursor + ramp).clamp(max=499)])
        K.step_map(cached, new, window, table, max_tokens=S + 3, out=out)
        cached.copy_(out.seq_lens)
        cursor.add_(out.used[1:].long())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                   # warms up, and is the first step
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    want, lens, at = np.array(table0), list(start), 0
    for it in range(30):
        if it:
            g.replay()
        torch.cuda.synchronize()
        lens, cu, slots, pos, used, want = fp8.step_map(lens, [1] * S, list(range(500))[at:], want,
                                                        S + 3)
        at += used[1]
        assert out.seq_lens.tolist() == lens and int(cursor) == at
        assert out.slot_mapping.tolist() == slots and out.positions.tolist() == pos
        assert np.array_equal(table.cpu().numpy(), want)
        (torch.ones(1000, device="cuda") * 2).sum().item()   # the program's own work between


@pytest.mark.parametrize("S,MB,hi,T", [
    (4097, 5, 9, 3000),    # the budget ends in the first of three tiles of requests
    (4097, 5, 9, 7000),    # in the second
    (9001, 3, 6, 5000),    # tiles behind it are granted nothing
    (9001, 3, 6, 17000),   # in the last
    (2049, 5, 9, 0), (2049, 5, 9, 1),
])
def test_budgets_that_end_inside_a_later_tile(S, MB, hi, T):
    cached, new, free, table = _random(S + T, S, MB, hi)
    room = np.minimum(new, MB * 16 - cached)
    assert room.sum() > T
    say("step map: budget", S, MB, hi, T, "of", int(room.sum()))
    _check(cached, new, free, table, T)
    _check(cached, new, free[:T // 64], table, T)      # and too few ids
