"""Pins of the fp64 definitions of the operators on packed sequences: closed forms,
invariances, and one operator written as another."""
import numpy as np
import pytest

from oracle import sequence_oracle as Q
from oracle import trackfit_oracle as O


def test_norm_has_unit_mean_square_and_rotation_keeps_it():
    r = np.random.default_rng(0)
    x = r.normal(size=(7, 3, 24)) * 5
    y = Q.qk_norm(x, None, 1e-12, positions=r.integers(0, 1000, 7), rot_dim=16)
    np.testing.assert_allclose(np.mean(y * y, -1), 1.0, rtol=1e-9)


def test_rotated_products_depend_on_the_distance_of_positions_alone():
    r = np.random.default_rng(1)
    q, k = r.normal(size=(1, 1, 32)), r.normal(size=(1, 1, 32))
    def product(pq, pk):
        a = Q.qk_norm(q, None, 1e-6, positions=[pq], rot_dim=32)
        b = Q.qk_norm(k, None, 1e-6, positions=[pk], rot_dim=32)
        return float(np.sum(a * b))
    assert abs(product(7, 3) - product(104, 100)) < 1e-12
    assert abs(product(7, 3) - product(7, 4)) > 1e-6


def test_rotation_at_position_zero_and_a_quarter_turn():
    x = np.arange(1.0, 17.0).reshape(1, 1, 16)
    plain = Q.qk_norm(x, None, 1e-6)
    np.testing.assert_array_equal(Q.qk_norm(x, None, 1e-6, positions=[0], rot_dim=16), plain)
    # base 1: all pairs turn by the position itself, in radians
    y = Q.qk_norm(x, None, 1e-6, positions=[1], rot_dim=16, rot_base=1.0)
    np.testing.assert_allclose(y[..., :8], plain[..., :8] * np.cos(1) - plain[..., 8:] * np.sin(1), rtol=1e-14)


def test_linear_attention_without_decay_is_causal_attention_without_softmax():
    r = np.random.default_rng(2)
    q, k, v = r.normal(size=(9, 2, 8)), r.normal(size=(9, 2, 8)), r.normal(size=(9, 2, 16))
    o, s = Q.linear_attention(q, k, v, np.zeros((9, 2)), [0, 9], 0.5)
    for h in range(2):
        np.testing.assert_allclose(o[:, h], 0.5 * np.tril(q[:, h] @ k[:, h].T) @ v[:, h], rtol=1e-12)
        np.testing.assert_allclose(s[0, h], k[:, h].T @ v[:, h], rtol=1e-12)


def test_linear_attention_goes_on_from_its_state_and_a_step_is_a_row():
    r = np.random.default_rng(3)
    q, k, v = r.normal(size=(11, 2, 8)), r.normal(size=(11, 2, 8)), r.normal(size=(11, 2, 8))
    g = -r.random((11, 2))
    o, s = Q.linear_attention(q, k, v, g, [0, 11])
    o1, s1 = Q.linear_attention(q[:10], k[:10], v[:10], g[:10], [0, 10])
    o2, s2 = Q.linear_attention_step(q[10:], k[10:], v[10:], g[10:], s1)
    np.testing.assert_allclose(np.concatenate([o1, o2]), o, rtol=1e-13)
    np.testing.assert_allclose(s2, s, rtol=1e-13)


def test_linear_attention_reversed_is_the_mirrored_sequence():
    r = np.random.default_rng(4)
    q, k, v, g = r.normal(size=(6, 1, 8)), r.normal(size=(6, 1, 8)), r.normal(size=(6, 1, 8)), -r.random((6, 1))
    o, s = Q.linear_attention(q, k, v, g, [0, 6], reverse=True)
    m, t = Q.linear_attention(q[::-1], k[::-1], v[::-1], g[::-1], [0, 6])
    np.testing.assert_array_equal(o, m[::-1])
    np.testing.assert_array_equal(s, t)


def test_linear_attention_with_one_key_channel_is_the_gated_scan():
    """K = 1, q = 1, k = z: S_t = (1 - z) S_{t-1} + z n, Eq. 2 with one gate a row."""
    r = np.random.default_rng(5)
    z, n = r.random((8, 1)), r.normal(size=(8, 5))
    ones = np.ones((8, 1, 1))
    o, _ = Q.linear_attention(ones, z[:, :, None], n[:, None, :], np.log1p(-z), [0, 8])
    h = np.zeros(5)
    for t in range(8):
        h = h + z[t] * (n[t] - h)
        np.testing.assert_allclose(o[t, 0], h, rtol=1e-12)


def test_a_decay_of_minus_infinity_forgets():
    r = np.random.default_rng(6)
    q, k, v = r.normal(size=(4, 1, 8)), r.normal(size=(4, 1, 8)), r.normal(size=(4, 1, 8))
    g = np.zeros((4, 1))
    g[2] = -np.inf
    o, _ = Q.linear_attention(q, k, v, g, [0, 4])
    p, _ = Q.linear_attention(q[2:], k[2:], v[2:], np.zeros((2, 1)), [0, 2])
    np.testing.assert_allclose(o[2:], p, rtol=1e-14)


@pytest.mark.parametrize("heads", [1, 2])
def test_cross_attention_of_a_sequence_to_itself_is_the_models_attention(heads):
    r = np.random.default_rng(7)
    n, d = 5, 16
    qkv = r.normal(size=(1, n, 3 * d))
    a = O.attention(*np.split(qkv, 3, axis=2), np.ones((1, n), bool), heads)
    q, k, v = (qkv[0, :, i * d:(i + 1) * d].reshape(n, heads, d // heads) for i in range(3))
    o = Q.cross_attention(q, k, v, [0, n], [0, n], (d // heads) ** -0.5)
    np.testing.assert_allclose(o.reshape(n, d), a[0], rtol=1e-12)


def test_cross_attention_without_states_is_zero_and_shared_heads_repeat():
    r = np.random.default_rng(8)
    q, k, v = r.normal(size=(5, 4, 8)), r.normal(size=(7, 2, 8)), r.normal(size=(7, 2, 8))
    o = Q.cross_attention(q, k, v, [0, 2, 5], [0, 0, 7], 0.3)
    assert np.all(o[:2] == 0)
    full = Q.cross_attention(q, np.repeat(k, 2, 1), np.repeat(v, 2, 1), [0, 2, 5], [0, 0, 7], 0.3)
    np.testing.assert_array_equal(o, full)
