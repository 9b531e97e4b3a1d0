"""Pins of oracle/longcontext.py: hand values, invariants, brute force."""
import math

import numpy as np
import pytest

from oracle import longcontext as lc
from oracle.attention import dense_attention


def test_frequencies_by_hand():
    assert np.allclose(lc.frequencies(4, 100.0), [1.0, 0.1], rtol=1e-15)
    assert np.allclose(lc.frequencies(4, 100.0, factor=4.0), [0.25, 0.025], rtol=1e-15)
    # over 20 pi tokens the pairs turn 10 times and once: with the line from 1 to 10 turns the first keeps, the second is divided
    f = lc.frequencies(4, 100.0, factor=4.0, original_len=20 * math.pi, low_turns=1.0, high_turns=10.0)
    assert np.allclose(f, [1.0, 0.025], rtol=1e-12)
    f = lc.frequencies(4, 100.0, factor=4.0, original_len=20 * math.pi, low_turns=0.0, high_turns=2.0)
    assert np.allclose(f, [1.0, 0.5 * 0.1 + 0.5 * 0.025], rtol=1e-12)


@pytest.mark.parametrize("layout,pair", [("halves", (1, 4)), ("interleaved", (2, 3))])
def test_a_quarter_turn_by_hand(layout, pair):
    x = np.arange(1.0, 9.0).reshape(1, 1, 8)
    freq = np.array([0.0, math.pi / 2, 0.0])                # six of eight elements, the second pair turns a quarter per position
    a, b = pair
    y = lc.turn(x, [1], freq, layout)[0, 0]
    want = x[0, 0].copy()
    want[a], want[b] = -x[0, 0, b], x[0, 0, a]
    assert np.allclose(y, want, atol=1e-15)
    assert np.allclose(lc.turn(x, [0], freq, layout, 2.0)[0, 0], np.concatenate([2 * x[0, 0, :6], x[0, 0, 6:]]))


@pytest.mark.parametrize("layout", ["halves", "interleaved"])
def test_logits_depend_on_distances_only(layout):
    r = np.random.default_rng(0)
    q, k = r.standard_normal((2, 1, 3, 16))
    f = lc.frequencies(12)
    dot = lambda p, s: (lc.turn(q, [p], f, layout) * lc.turn(k, [s], f, layout)).sum(-1)  # noqa: E731
    assert np.allclose(dot(7, 3), dot(1007, 1003), atol=1e-9) and not np.allclose(dot(7, 3), dot(7, 4), atol=1e-3)
    assert np.allclose(lc.turn(lc.turn(q, [9], f, layout), [-9], f, layout), q)


def test_scores_bound_every_key():
    r = np.random.default_rng(1)
    q, K = r.standard_normal((4, 32)), r.standard_normal((80, 1, 32))
    s = lc.scores(q, lc.page_bounds(K)[:, 0])
    logits = (q @ K[:, 0].T).sum(0)
    for p in range(5):
        assert logits[16 * p:16 * p + 16].max() <= s[p] + 1e-5
    brute = [sum(max(qh[d] * K[16 * p:16 * p + 16, 0, d].min(), qh[d] * K[16 * p:16 * p + 16, 0, d].max()) for qh in q for d in range(32)) for p in range(5)]
    assert np.allclose(s, brute, rtol=1e-6)


def test_choice_by_hand():
    s = np.array([9, 1, 5, np.nan, 5, 5, 0, 9], np.float32)
    assert lc.choose(s, 8, 8, 1, 1) == list(range(8))
    assert lc.choose(s, 8, 5, 1, 2) == [0, 2, 3, 6, 7]      # NaN first, then the first of the three fives
    assert lc.choose(s, 8, 6, 1, 2) == [0, 2, 3, 4, 6, 7]
    assert lc.choose(s, 8, 3, 1, 2) == [0, 6, 7]
    assert lc.choose(s, 8, 2, 0, 1) == [3, 7]


def test_a_budget_for_everything_is_dense_attention():
    r = np.random.default_rng(2)
    q, K, V = r.standard_normal((3, 4, 8)), r.standard_normal((50, 2, 8)), r.standard_normal((50, 2, 8))
    out, picked = lc.sparse_attention(q, K, V, 47, 4, 1, 1)
    assert np.allclose(out, dense_attention(q, K, V, 47, dtype=np.float64)) and picked[0] == [[0, 1, 2], [0, 1, 2]]
    out, picked = lc.sparse_attention(q, K, V, 47, 2, 1, 1)
    assert picked[2] == [[0, 3], [0, 3]]
    K2, V2 = (np.concatenate([x[:16], x[48:50]]) for x in (K, V))
    assert np.allclose(out[2], dense_attention(q[2:], K2, V2, 17, dtype=np.float64)[0])
