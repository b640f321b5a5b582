"""Drafted trees, accepted paths, running weights and evicted contexts on a handle, against the oracle.

Hidden states are held to the tolerances of every decode test.  A running weight's relative error is twice its score's absolute
error: q and k are rounded to fp16 (2^-11 relative each) from projections of operands rounded to fp16 (the same again), so at most
4 * 2^-11 * sum |q k| / sqrt(hd) plus, from the second layer on, what the hidden states' own error moves (held to 1 %).
"""
import numpy as np
import pytest

from oracle import cache_ops as ops
from oracle import decode_tree as dt
from oracle import reuse_prefill as orc
from paper_2601_11553_b200 import percache as pcb
from paper_2601_11553_b200 import workloads as wl
from tests import gpu_helpers as G
from tests import helpers as H

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, seed, spec, reserve, n_layers=2, flags=0, **kw):
        ws = [wl.small_workload(seed=seed, n_layers=n_layers, chunk_lens=cl, n_query=nq, hit_idx=hi, id_base=100 + 50 * b, **kw)
              for b, (cl, nq, hi) in enumerate(spec)]
        self.seed, self.shape = seed, ws[0].shape
        self.weights = wl.make_weights(self.shape, seed, random_gains=True)
        self.model = H.oracle_model(self.shape, self.weights)
        self.prompts = [w.prompts[0] for w in ws]
        cached = [c for w in ws for c in w.cached_ids]
        lens = {c: n for p in self.prompts for c, n in zip(p.chunk_ids, p.chunk_len)}
        store = G.oracle_store_alone(self.model, seed, [(c, lens[c]) for c in cached])
        want = orc.reuse_prefill(self.model, store, [H.oracle_prompt(p, [i for i, c in enumerate(p.chunk_ids) if c in cached])
                                                     for p in self.prompts], keep_ctx=True, commit=False)
        self.states = [dt.begin(r) for r in want]
        self.h = G.make_handle(self.shape, self.weights, self.prompts, decode_reserve=reserve, flags=flags,
                               pool_pages=sum(-(-x // 16) for p in self.prompts for x in p.chunk_len) + 64 + 8 * len(spec))
        self.h.set_decode_reserve(reserve)
        G.push_store(self.h, store, cached)
        self.h.prefill(G.specs_for(self.prompts, cached))
        self.n = 0

    def tokens(self, rows):
        self.n += 1
        return wl.make_hidden(self.seed, (9, 1000 * self.n), max(rows, 1), self.shape.d_model)[:rows]

    def close_to(self, got, want):
        c = G.compare_hidden(got, want)
        assert c["max_abs"] <= G.TOL_MAX_ABS and c["mean_abs"] <= G.TOL_MEAN_ABS, c

    def tree(self, parents):
        """One decode_tree call, checked; returns the tokens per prompt."""
        bits = self.tokens(sum(len(p) for p in parents))
        got = self.h.decode_tree(parents, np.ascontiguousarray(bits))
        hidden, at = [], 0
        for b, p in enumerate(parents):
            hidden.append(orc.bf16_bits_to_f64(bits[at:at + len(p)]))
            if len(p):
                self.close_to(got[at:at + len(p)], dt.tree_outputs(self.model, self.states[b], p, hidden[b]))
            at += len(p)
        return hidden

    def accept(self, hidden, paths, track=False, decay=1.0):
        self.h.accept(paths)
        for b, p in enumerate(paths):
            dt.accept(self.model, self.states[b], hidden[b], p, track, decay)

    def decode(self, track=False, decay=1.0):
        bits = self.tokens(len(self.prompts))
        got = self.h.decode(np.ascontiguousarray(bits))
        want = []
        for b, st in enumerate(self.states):
            y, share = dt.step(self.model, st, orc.bf16_bits_to_f64(bits[b]))
            want.append(y)
            if track:
                for l in range(self.shape.n_layers):
                    st.w[l] = decay * st.w[l] + share[l]
        self.close_to(got, np.stack(want))

    def check_context(self):
        for b, st in enumerate(self.states):
            for l in range(self.shape.n_layers):
                k, v = self.h.read_ctx(b, l, st.k[l].shape[0])
                assert np.max(np.abs(k.astype(np.float64) - st.k[l].reshape(len(k), -1))) < 3e-2
                assert np.max(np.abs(v.astype(np.float64) - st.v[l].reshape(len(v), -1))) < 3e-2

    def check_weights(self):
        for b, st in enumerate(self.states):
            rel = 8 * 2.0 ** -11 * st.score_abs + 0.01
            for l in range(self.shape.n_layers):
                w = self.h.read_weights(b, l, st.k[l].shape[0], self.shape.n_kv_heads)
                assert w.shape == st.w[l].shape
                assert (np.abs(w - st.w[l]) <= rel * st.w[l] + 1e-7).all(), (b, l, np.abs(w - st.w[l]).max())


BRANCHY = [-1, 0, 0, 1, 1, 2, 5, -1, 7]


@pytest.mark.parametrize("kw", [dict(), dict(n_q_heads=8, n_kv_heads=2, d_model=512), dict(flags=pcb.FLAG_SINGLE_CTA_GEMM)])
def test_trees_accepted_paths_and_plain_tokens_in_turn(kw):
    c = Case(71, [([128, 100, 160], 40, [0, 2]), ([60], 7, [])], reserve=24, **kw)
    with c.h:
        hidden = c.tree([BRANCHY, [-1, 0, 1]])
        c.accept(hidden, [[0, 2, 5, 6], []])
        c.check_context()
        c.decode()                                       # the streaming kernels, on the context the path has become part of
        hidden = c.tree([[-1], BRANCHY])
        c.accept(hidden, [[0], [7, 8]])
        c.check_context()
        c.tree([[-1, -1], [-1]])                         # not accepted: dropped
        c.decode()
        c.tree([[], [-1, 0]])                            # a prompt may sit a step out
        c.check_context()


def test_a_tree_of_64_nodes_and_one_of_200():
    c = Case(72, [([200], 9, [0])], reserve=210, n_layers=1)
    rng = np.random.default_rng(3)
    with c.h:
        hidden = c.tree([[int(rng.integers(-1, i)) if i else -1 for i in range(64)]])
        c.accept(hidden, [[0]])
        parents = [i - 1 if i < 70 else int(rng.integers(0, 70)) for i in range(200)]
        hidden = c.tree([parents])
        c.accept(hidden, [dt.path_to(parents, 69)])
        c.check_context()


def test_trees_after_a_gather_free_prefill():
    c = Case(73, [([512, 256], 16, [0, 1]), ([640], 5, [0])], reserve=16, flags=pcb.FLAG_GATHER_FREE)
    with c.h:
        assert c.h.stats()["gather_free"] == 1
        hidden = c.tree([BRANCHY, [-1, 0]])
        c.accept(hidden, [[0, 1, 4], [0, 1]])
        c.check_context()
        c.decode()


def test_running_weights_and_eviction():
    c = Case(74, [([128, 60], 20, [0]), ([40], 9, []), ([300], 3, [0])], reserve=24, flags=pcb.FLAG_TRACK_WEIGHTS)
    hkv = c.shape.n_kv_heads
    with c.h:
        c.h.set_weight_decay(0.75)
        c.decode(track=True, decay=0.75)
        c.decode(track=True, decay=0.75)
        c.check_weights()
        hidden = c.tree([BRANCHY, [-1, 0], [-1]])
        c.accept(hidden, [[0, 2, 5], [], [0]], track=True, decay=0.75)
        # a prompt whose path is empty decays all the same
        for l in range(c.shape.n_layers):
            c.states[1].w[l] *= 0.75
        c.check_weights()
        c.tree([[-1], [], [-1]])
        c.h.accept([[], [], []])                         # nothing kept: one more decay, nothing else
        for st in c.states:
            for l in range(c.shape.n_layers):
                st.w[l] *= 0.75
        c.check_context()
        c.check_weights()
        for budget, sink, recent in ((100, 2, 16), (40, 0, 40), (33, 4, 0)):
            slots = [st.k[0].shape[0] for st in c.states]
            w = [[c.h.read_weights(b, l, slots[b], hkv) for l in range(c.shape.n_layers)] for b in range(3)]
            before = [[c.h.read_ctx(b, l, slots[b]) for l in range(c.shape.n_layers)] for b in range(3)]
            c.h.evict_context(budget, sink, recent)
            for b in range(3):
                n = min(slots[b], budget)
                for l in range(c.shape.n_layers):
                    k, v = c.h.read_ctx(b, l, n)
                    left = c.h.read_weights(b, l, n, hkv)
                    assert left.shape == (hkv, n)
                    for g in range(hkv):                 # exactly the slots that the library's own weights choose
                        at = ops.select_slots(w[b][l][g], slots[b], budget, sink, recent)
                        cols = slice(g * 128, (g + 1) * 128)
                        assert np.array_equal(k[:, cols], before[b][l][0][at][:, cols]) and np.array_equal(v[:, cols], before[b][l][1][at][:, cols])
                        assert np.array_equal(left[g], w[b][l][g, at])
                dt.evict(c.states[b], budget, sink, recent, w[b])
            c.check_context()
            c.check_weights()
            c.decode(track=True, decay=0.75)             # positions go on where they were
            hidden = c.tree([[-1, 0, 1], [-1, -1], [-1, 0]])
            c.accept(hidden, [[0, 1], [1], [0, 1]], track=True, decay=0.75)
            c.check_context()
            c.check_weights()


def test_a_context_cut_to_its_budget_leaves_room_for_more_tokens():
    c = Case(75, [([64], 8, [])], reserve=4, n_layers=1, flags=pcb.FLAG_TRACK_WEIGHTS)
    with c.h:
        for _ in range(4):
            c.decode(track=True)
        with pytest.raises(pcb.PerCacheError) as e:
            c.h.decode(np.ascontiguousarray(c.tokens(1)))
        assert e.value.code == pcb.E_CAPACITY
        w = [c.h.read_weights(0, 0, 76, c.shape.n_kv_heads)]
        c.h.evict_context(50, 1, 8)
        dt.evict(c.states[0], 50, 1, 8, w)
        with pytest.raises(pcb.PerCacheError) as e:      # there are slots, but no positions: max_prompt_tokens is 76
            c.h.decode(np.ascontiguousarray(c.tokens(1)))
        assert e.value.code == pcb.E_CAPACITY
        c.check_context()


def test_refusals_change_nothing():
    c = Case(76, [([64], 8, []), ([32], 4, [])], reserve=8, n_layers=1)

    def refused(code, fn, *a):
        with pytest.raises(pcb.PerCacheError) as e:
            fn(*a)
        assert e.value.code == code

    with c.h:
        tok = lambda n: np.ascontiguousarray(c.tokens(n))          # noqa: E731
        refused(pcb.E_INVAL, c.h.accept, [[0], [0]])               # no tree
        refused(pcb.E_INVAL, c.h.decode_tree, [[-1]], tok(1))      # one prompt of two
        refused(pcb.E_INVAL, c.h.decode_tree, [[], []], tok(0))
        refused(pcb.E_INVAL, c.h.decode_tree, [[0], [-1]], tok(2))         # a parent behind its child
        refused(pcb.E_INVAL, c.h.decode_tree, [[-1, -2], [-1]], tok(3))
        refused(pcb.E_INVAL, c.h.decode_tree, [[-1] * 257, [-1]], tok(258))
        refused(pcb.E_CAPACITY, c.h.decode_tree, [[-1] * 9, [-1]], tok(10))
        refused(pcb.E_INVAL, c.h.evict_context, 16)                # nothing tracked
        refused(pcb.E_INVAL, c.h.set_weight_decay, -1.0)
        refused(pcb.E_INVAL, c.h.set_weight_decay, float("nan"))
        hidden = c.tree([[-1, 0, 0], [-1]])
        refused(pcb.E_INVAL, c.h.accept, [[1], [0]])               # starts below a root
        refused(pcb.E_INVAL, c.h.accept, [[0, 1, 2], [0]])         # not a path
        refused(pcb.E_INVAL, c.h.accept, [[0, 3], [0]])
        refused(pcb.E_INVAL, c.h.accept, [[0]])
        c.accept(hidden, [[0, 2], [0]])
        refused(pcb.E_INVAL, c.h.accept, [[0], [0]])               # accepted already
        c.check_context()
        c.decode()
        c.h.set_flags(pcb.FLAG_TRACK_WEIGHTS)
        c.decode(track=True)
        refused(pcb.E_INVAL, c.h.evict_context, 16, 9, 8)
        refused(pcb.E_INVAL, c.h.evict_context, 0)
        hidden = c.tree([[-1], [-1]])
        refused(pcb.E_INVAL, c.h.evict_context, 16)                # a tree is waiting
        c.accept(hidden, [[0], [0]], track=True)
        c.check_context()
        c.check_weights()


def test_a_refused_step_leaves_the_nodes_to_be_accepted():
    c = Case(77, [([64], 8, []), ([32], 4, [])], reserve=3, n_layers=1)
    with c.h:
        c.accept(c.tree([[-1, 0, 1], [-1]]), [[0, 1, 2], []])          # the first prompt's reserve is used up
        hidden = c.tree([[], [-1, 0]])
        with pytest.raises(pcb.PerCacheError) as e:
            c.h.decode(np.ascontiguousarray(c.tokens(2)))
        assert e.value.code == pcb.E_CAPACITY
        c.accept(hidden, [[], [0, 1]])
        c.check_context()


@pytest.mark.parametrize("flags", [0, pcb.FLAG_TRACK_WEIGHTS])
def test_a_reserve_set_after_the_prefill_holds_from_the_next_one(flags):
    c = Case(78, [([64], 8, []), ([32], 4, [])], reserve=2, n_layers=1, flags=flags)
    with c.h:
        c.h.set_decode_reserve(50)
        for _ in range(2):
            c.decode(track=bool(flags))
        for call, arg in ((c.h.decode, 2), (lambda x: c.h.decode_tree([[-1], []], x), 1)):
            with pytest.raises(pcb.PerCacheError) as e:
                call(np.ascontiguousarray(c.tokens(arg)))
            assert e.value.code == pcb.E_CAPACITY
        c.check_context()
