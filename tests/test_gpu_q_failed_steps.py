"""What a step on a handle's context leaves behind when one of its launches fails half-way (made on the host)."""
import numpy as np
import pytest

from paper_2601_11553_b200 import percache as pcb
from tests.test_gpu_n_decode_tree import Case

pytestmark = pytest.mark.gpu


def fails(call, *args):
    with pytest.raises(pcb.PerCacheError) as e:
        call(*args)
    assert e.value.code == pcb.E_CUDA


def sums_are_gone(c):
    for call in (lambda: c.h.evict_context(16), lambda: c.h.read_weights(0, 0, 200, c.shape.n_kv_heads)):
        with pytest.raises(pcb.PerCacheError) as e:
            call()
        assert e.value.code == pcb.E_INVAL
    for st in c.states:
        for l in range(c.shape.n_layers):
            st.w[l] *= 0


@pytest.mark.parametrize("layer", [0, 1, 2])
def test_a_failed_tracked_token_ends_the_running_weights(layer):
    c = Case(81, [([64], 8, []), ([32], 4, [])], reserve=8, n_layers=3, flags=pcb.FLAG_TRACK_WEIGHTS)
    with c.h:
        c.decode(track=True)
        c.h.fail_layer(layer)
        fails(c.h.decode, np.ascontiguousarray(c.tokens(2)))
        sums_are_gone(c)
        c.check_context()
        c.decode(track=True)                             # the sums start again from zero
        c.check_weights()
        c.decode(track=True)
        c.check_weights()
        c.check_context()


@pytest.mark.parametrize("layer", [0, 1, 2])
def test_a_failed_accept_drops_the_nodes_and_ends_the_running_weights(layer):
    c = Case(82, [([64], 8, []), ([32], 4, [])], reserve=12, n_layers=3, flags=pcb.FLAG_TRACK_WEIGHTS)
    with c.h:
        c.decode(track=True)
        c.tree([[-1, 0, 0, 2], [-1, -1]])
        c.h.fail_layer(layer)
        fails(c.h.accept, [[0, 2, 3], [1]])
        sums_are_gone(c)
        c.check_context()
        with pytest.raises(pcb.PerCacheError) as e:
            c.h.accept([[0], [1]])
        assert e.value.code == pcb.E_INVAL
        # later tokens take the slots that the nodes' weights were for
        hidden = c.tree([[-1, 0], [-1]])
        c.accept(hidden, [[0, 1], [0]], track=True)
        c.check_weights()
        c.decode(track=True)
        c.check_weights()
        c.check_context()


def test_a_failed_tree_step_keeps_the_running_weights():
    c = Case(83, [([64], 8, []), ([32], 4, [])], reserve=12, n_layers=2, flags=pcb.FLAG_TRACK_WEIGHTS)
    with c.h:
        c.decode(track=True)
        c.h.fail_layer(1)
        fails(c.h.decode_tree, [[-1, 0], [-1]], np.ascontiguousarray(c.tokens(3)))
        c.check_weights()
        c.check_context()
        c.decode(track=True)
        c.check_weights()


def test_a_failed_eviction_ends_the_batch():
    c = Case(84, [([64], 8, []), ([32], 4, [])], reserve=12, n_layers=2, flags=pcb.FLAG_TRACK_WEIGHTS)
    with c.h:
        c.decode(track=True)
        c.h.fail_layer(1)
        fails(c.h.evict_context, 16)
        with pytest.raises(pcb.PerCacheError) as e:
            c.h.decode(np.ascontiguousarray(c.tokens(2)))
        assert e.value.code == pcb.E_INVAL
