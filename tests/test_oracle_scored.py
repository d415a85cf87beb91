"""The oracle of capped, biased and windowed scores, pinned by closed forms, brute force and
the plain oracle."""
import numpy as np
import pytest

import oracle
from oracle.scored import scored_attention, scores
from workloads import make_batch_from_lens


def _batch(lens, new, seed=0, hq=4, hkv=2, d=64):
    return make_batch_from_lens(lens, new, dtype="bf16", num_q_heads=hq, num_kv_heads=hkv,
                                head_dim=d, block_size=16, seed=seed, keep_contig=True)


def _run(b, **kw):
    return scored_attention(b.q_raw(), b.kv_raw(), b.block_table, b.seq_lens, b.cu_seqlens_q,
                            dtype=b.dtype, num_q_heads=b.num_q_heads, num_kv_heads=b.num_kv_heads,
                            head_dim=b.head_dim, scale=b.scale, **kw)


def test_without_any_it_is_the_plain_one():
    b = _batch([40, 1, 70], [7, 1, 70])
    want = oracle.paged_attention(b.q_raw(), b.kv_raw(), b.block_table, b.seq_lens,
                                  b.cu_seqlens_q, dtype="bf16", num_q_heads=4, num_kv_heads=2,
                                  head_dim=64, block_size=16, scale=b.scale)
    out, weight = _run(b)
    assert np.allclose(out, want, atol=1e-12)
    assert (weight >= np.abs(out) - 1e-12).all()
    for kw in (dict(window=70), dict(window=10 ** 6), dict(softcap=1e9),
               dict(slopes=np.zeros(4))):
        assert np.allclose(_run(b, **kw)[0], want, atol=1e-6), kw


def test_scores_by_hand():
    q, k = np.array([[2.0]]), np.array([[1.0], [3.0], [5.0]])
    a = scores(q, k, np.array([2]), np.arange(3), scale=0.5, softcap=2.0, slope=0.25, window=2)
    assert a[0, 0] == -np.inf
    assert np.allclose(a[0, 1:], [2 * np.tanh(1.5) - 0.25, 2 * np.tanh(2.5)])


def test_a_window_of_one_gives_each_row_its_own_value():
    b = _batch([50], [20])
    out, _ = _run(b, window=1)
    v = b.v_contig[0].double().numpy()[30:]
    assert np.allclose(out, np.repeat(v, 2, 1))


@pytest.mark.parametrize("window", [3, 16, 17, 40])
def test_a_window_is_attention_over_its_tokens(window):
    """Brute force over every row, keys taken one by one."""
    b = _batch([61], [25], seed=window)
    out, _ = _run(b, window=window, softcap=1.5, slopes=[0.1, 0.2, -0.1, 0])
    q, k, v = (x.double().numpy() for x in (b.q, b.k_contig[0], b.v_contig[0]))
    for i in range(25):
        p = 36 + i
        for h in range(4):
            t = [t for t in range(61) if p - window < t <= p]
            a = [1.5 * np.tanh(b.scale * float(q[i, h] @ k[x, h // 2]) / 1.5) +
                 [0.1, 0.2, -0.1, 0][h] * (x - p) for x in t]
            w = np.exp(a) / np.exp(a).sum()
            assert np.allclose(out[i, h], sum(y * v[x, h // 2] for x, y in zip(t, w)))


def test_what_no_row_sees_is_not_looked_at():
    b = _batch([100], [3])
    want, _ = _run(b, window=20)           # rows at 97 .. 99 see 78 on: block 4 from slot 14 on
    b.block_table[0, :4] = -1
    assert np.array_equal(_run(b, window=20)[0], want)
    b.block_table[0, 0] = 10 ** 6
    assert np.array_equal(_run(b, window=20)[0], want)


def test_a_steep_slope_leaves_the_nearest_key():
    b = _batch([30], [1])
    out, _ = _run(b, slopes=[80.0] * 4)
    assert np.allclose(out[0], np.repeat(b.v_contig[0].double().numpy()[29], 2, 0), atol=1e-9)


def test_a_low_cap_makes_weights_equal():
    b = _batch([30], [1])
    out, _ = _run(b, softcap=1e-9)
    assert np.allclose(out[0], np.repeat(b.v_contig[0].double().numpy().mean(0), 2, 0), atol=1e-7)


def test_an_empty_sequence_gives_zeros():
    b = _batch([20, 20], [1, 1])
    b.seq_lens[1] = 0
    out, weight = _run(b, softcap=3.0)
    assert not out[1].any() and not weight[1].any() and out[0].any()
