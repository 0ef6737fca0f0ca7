"""Pins of the float64 reference of norm, rotary positions and attention (oracle/layer_oracle.py): closed forms and brute force."""
import math

import numpy as np
import pytest

from oracle import layer_oracle as o


def test_norm_of_a_row_by_hand():
    x = np.array([[3.0, 4.0]])
    h, y = o.rms_norm(x, np.array([1.0, 2.0]), 0.0)
    assert np.allclose(y, [[3 / math.sqrt(12.5), 8 / math.sqrt(12.5)]], atol=1e-15) and np.array_equal(h, x)
    h, y = o.rms_norm(x, np.ones(2), 0.0, residual=np.array([[-3.0, -4.0 + 1e-3]]))
    assert np.allclose(y, [[0.0, math.sqrt(2)]], atol=1e-12)            # the norm is of the sum
    assert np.allclose(o.rms_norm(np.zeros((1, 4)), np.ones(4), 1e-5)[1], 0.0)


def test_frequencies_and_their_stretching():
    assert np.allclose(o.rope_frequencies(4, base=100.0), [1.0, 0.1])
    assert np.allclose(o.rope_frequencies(4, base=100.0, factor=4.0), [0.25, 0.025])
    # a trained length of 40: wave 0 turns 40 / 2 pi = 6.4 times (stays), wave 1 0.64 times (stretched in full)
    assert np.allclose(o.rope_frequencies(4, base=100.0, factor=4.0, trained=40.0, low=1.0, high=4.0), [1.0, 0.025])
    turns = 15 / (2 * math.pi)
    keep = (turns - 1) / 3
    assert np.allclose(o.rope_frequencies(4, base=100.0, factor=4.0, trained=15.0)[0], keep + (1 - keep) / 4)


@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_keeps_relative_positions(pairs):
    """q(p) . k(t) depends on p - t alone, and a part that does not turn stays."""
    rng = np.random.default_rng(3)
    q, k = rng.standard_normal((2, 1, 12))
    w = o.rope_frequencies(8)
    dots = [float((o.rotate(q, w * p, pairs) @ o.rotate(k, w * (p - 5), pairs).T)[0, 0]) for p in (5, 17, 300)]
    assert np.allclose(dots, dots[0], atol=1e-12)
    assert np.array_equal(o.rotate(q, w * 9, pairs)[:, 8:], q[:, 8:])
    quarter = o.rotate(np.array([[1.0, 0, 0, 0]]), np.array([math.pi / 2, 0.0]), pairs)
    assert np.allclose(quarter, [[0, 1, 0, 0]] if pairs else [[0, 0, 1, 0]])


def test_attention_by_brute_force():
    rng = np.random.default_rng(4)
    K, V = rng.standard_normal((2, 5, 2, 4, 3))
    table = np.array([[3, 1], [4, 0]])
    row_start, kv_len = [0, 2, 5], [6, 2]
    Q = rng.standard_normal((5, 4 * 3))
    O, A = o.attention(Q, K, V, 4, row_start, kv_len, table, 0.7, True)
    for row, s, seen in ((0, 0, 5), (1, 0, 6), (2, 1, 0), (3, 1, 1), (4, 1, 2)):
        for h in range(4):
            got = np.zeros(3)
            total = 0.0
            for p in range(seen):
                page = table[s][p // 4]
                e = math.exp(0.7 * float(np.dot(Q[row, 3 * h:3 * h + 3], K[page, h // 2, p % 4])))
                total += e
                got += e * V[page, h // 2, p % 4]
            assert np.allclose(O[row, 3 * h:3 * h + 3], got / total if seen else 0.0, atol=1e-12)
    assert np.all(A >= np.abs(O) - 1e-12)
    everything, _ = o.attention(Q, K, V, 4, row_start, kv_len, table, 0.7, False)
    assert np.allclose(everything[1], O[1]) and not np.allclose(everything[0], O[0])
    equal = o.attend(np.zeros(3), K[0, 0], V[0, 0], 1.0, 4)[0]
    assert np.allclose(equal, V[0, 0].mean(0))
