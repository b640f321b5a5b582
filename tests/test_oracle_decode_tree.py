"""Pins of the tree-decode oracle: to the plain decode oracle, and of its eviction by hand."""
import numpy as np

from oracle import decode as dec
from oracle import decode_tree as dt
from oracle import reuse_prefill as orc
from paper_2601_11553_b200 import workloads as wl
from tests import helpers as H


def _start(seed=5):
    w = wl.small_workload(seed=seed, n_layers=2, chunk_lens=[19, 8], n_query=5, hit_idx=[])
    model = H.oracle_model(w.shape, wl.make_weights(w.shape, seed, random_gains=True))
    res = orc.reuse_prefill(model, orc.Store(), [H.oracle_prompt(w.prompts[0], [])], keep_ctx=True, commit=False)[0]
    toks = orc.bf16_bits_to_f64(wl.make_hidden(seed, (9, 0), 6, w.shape.d_model))
    return model, res, toks


def test_a_chain_is_plain_decoding():
    model, res, toks = _start()
    plain, st = dec.begin_decode(res), dt.begin(res)
    tree = dt.tree_outputs(model, st, [-1, 0, 1], toks)
    for i in range(3):
        want = dec.decode_step(model, plain, toks[i])
        got, share = dt.step(model, st, toks[i])
        assert np.allclose(got, want, atol=1e-12) and np.allclose(tree[i], want, atol=1e-12)
        assert np.allclose(share[0].sum(1), model.n_q_heads // model.n_kv_heads)
    assert np.allclose(st.k[1], plain.k_ctx[1]) and st.position == plain.n_tokens


def test_siblings_start_from_the_same_context():
    model, res, toks = _start(6)
    st = dt.begin(res)
    out = dt.tree_outputs(model, st, [-1, -1, 0], toks)
    for i, path in enumerate(([0], [1], [0, 2])):
        s = dec.begin_decode(res)
        for j in path:
            y = dec.decode_step(model, s, toks[j])
        assert np.allclose(out[i], y, atol=1e-12)
    assert dt.path_to([-1, 0, 0, 2], 3) == [0, 2, 3]


def test_eviction_keeps_the_chosen_slots_of_every_head():
    model, res, toks = _start(7)
    st = dt.begin(res)
    dt.accept(model, st, toks, [0, 1], True, 0.5)
    assert np.allclose(sum(w.sum() for w in st.w), 2 * 2 * model.n_q_heads)
    k, n = st.k[0].copy(), st.k[0].shape[0]
    weights = [np.tile(np.arange(n)[::-1], (2, 1)).astype(float) for _ in st.k]
    weights[0][1] = np.arange(n)
    dt.evict(st, 5, 1, 1, weights)
    assert np.array_equal(st.k[0][:, 0], k[[0, 1, 2, 3, n - 1], 0])
    assert np.array_equal(st.k[0][:, 1], k[[0, n - 4, n - 3, n - 2, n - 1], 1])
    assert st.position == n
