"""Pins of the cache-operator oracle: closed forms, brute force, and consistency with a dense causal softmax."""
import numpy as np

from oracle import cache_ops as ops


def test_chain_equals_dense_causal_attention():
    rng = np.random.default_rng(1)
    t, n, hq, hkv, d = 11, 4, 4, 2, 8
    k, v = rng.standard_normal((t, hkv, d)), rng.standard_normal((t, hkv, d))
    q = rng.standard_normal((n, hq, d))
    out, lse, _ = ops.tree_attention(q, k, v, t - n, None, 0.3)
    for i in range(n):
        for h in range(hq):
            s = np.array([0.3 * q[i, h] @ k[j, h // 2] for j in range(t - n + i + 1)])
            p = np.exp(s) / np.exp(s).sum()
            assert np.allclose(out[i, h], sum(p[j] * v[j, h // 2] for j in range(len(p))), atol=1e-12)
            assert np.isclose(lse[i, h], np.log(np.exp(s).sum()))


def test_siblings_do_not_see_each_other_and_an_empty_row_is_zero():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((3, 1, 4)), rng.standard_normal((3, 1, 4))
    q = rng.standard_normal((3, 1, 4))
    mask = np.array([[1, 0, 0], [0, 1, 0], [0, 0, 0]], dtype=bool)
    out, lse, _ = ops.tree_attention(q, k, v, 0, mask, 1.0)
    assert np.allclose(out[0, 0], v[0, 0]) and np.allclose(out[1, 0], v[1, 0])          # one visible slot each
    assert np.array_equal(out[2], np.zeros((1, 4))) and lse[2, 0] == -np.inf


def test_weights_sum_to_rows_times_heads_and_decay():
    rng = np.random.default_rng(3)
    t, n, hq, hkv, d = 9, 3, 6, 2, 4
    k, v = rng.standard_normal((t, hkv, d)), rng.standard_normal((t, hkv, d))
    q = rng.standard_normal((n, hq, d))
    _, lse, _ = ops.tree_attention(q, k, v, t - n, None, 0.5)
    w0 = rng.random((hkv, t))
    w = ops.attention_weights(q, k, lse, None, t - n, None, 0.5, w0, 0.25)
    assert np.allclose((w - 0.25 * w0).sum(1), n * hq // hkv)
    one = ops.attention_weights(q, k, lse, [0, 1, 0], t - n, None, 0.5, w0, 0.0)
    assert np.allclose(one.sum(1), hq // hkv) and one[0, t - 1] == 0


def test_selection_by_hand():
    w = np.array([0.0, 5.0, 1.0, 1.0, np.nan, 1.0, -np.inf, 9.0])
    assert ops.select_slots(w, 8, 8, 0, 0) == list(range(8))
    assert ops.select_slots(w, 8, 3, 0, 0) == [1, 2, 7]               # ties: the lower slot
    assert ops.select_slots(w, 8, 4, 1, 2) == [0, 1, 6, 7]
    assert ops.select_slots(w, 7, 6, 0, 0) == [0, 1, 2, 3, 4, 5]      # NaN equals -inf: slot 4 before slot 6
    assert ops.select_slots(w, 7, 2, 0, 2) == [5, 6]
