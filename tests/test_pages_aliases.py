"""Operators on pages: arrays that are written must not overlap others of the call.  The addresses mean nothing and the device does not exist: an accepted
call ends at the device."""
import ctypes as C

import pytest

from paper_2601_11553_b200 import percache as pcb
from tests.test_ops_abi import lib       # noqa: F401

NO_DEVICE = 1 << 20
A = 1 << 30
N_SEQS, N_CHILDREN, WIDTH, WIDTH_OUT, PAGES = 2, 3, 8, 9, 100
INPUTS = {"page_table": N_SEQS * WIDTH, "held": N_SEQS, "length": N_SEQS, "parent": N_CHILDREN, "refs": PAGES, "free_list": PAGES, "free_count": 1}
OUTPUTS = {"table_out": N_CHILDREN * WIDTH_OUT, "held_out": N_CHILDREN, "length_out": N_CHILDREN, "refs_out": PAGES, "free_list_out": PAGES, "free_count_out": 1,
           "missing": 1}
AT = {name: A + 4096 * i for i, name in enumerate([*INPUTS, *OUTPUTS])}
WS = A + (1 << 26)


def fork(lib, ws=WS, **kw):                          # noqa: F811
    s = pcb.ForkStruct(N_SEQS, N_CHILDREN, WIDTH, WIDTH_OUT)
    s.n_pages, s.room = PAGES, 1
    for name, at in {**AT, **kw}.items():
        setattr(s, name, at)
    return lib.percache_fork_pages(NO_DEVICE, None, C.byref(s), ws, pcb.OPS_WORKSPACE_BYTES)


IN_PLACE = {name + "_out": AT[name] for name in ("refs", "free_list", "free_count")}


def test_arrays_apart_and_in_place_are_accepted(lib):        # noqa: F811
    assert fork(lib) == pcb.E_CUDA
    assert fork(lib, **IN_PLACE) == pcb.E_CUDA
    # inputs may be one array; arrays may lie one behind the other
    assert fork(lib, held=AT["length"], parent=AT["length"]) == pcb.E_CUDA
    assert fork(lib, held_out=AT["held"] + 4 * N_SEQS, length_out=AT["held"] + 4 * (N_SEQS + N_CHILDREN), missing=AT["held"] - 4) == pcb.E_CUDA
    # arrays without elements overlap nothing
    assert fork(lib, n_children=0, table_out=AT["page_table"], held_out=AT["held"], length_out=None) == pcb.E_CUDA


@pytest.mark.parametrize("out", [*OUTPUTS])
@pytest.mark.parametrize("other", [*INPUTS, *OUTPUTS])
def test_outputs_that_overlap_another_array_are_refused(lib, out, other):        # noqa: F811
    if out == other:
        return
    size = {**INPUTS, **OUTPUTS}[other]
    for place in (AT[other], AT[other] + 4 * (size - 1), AT[other] - 4 * (OUTPUTS[out] - 1)):
        in_place = out[:-4] == other and place == AT[other]
        if in_place:                                 # one of the three alone is refused for that
            assert fork(lib, **{**IN_PLACE, out: place + 4}) == pcb.E_INVAL
        assert fork(lib, **{out: place}) == pcb.E_INVAL, (out, other, place - AT[other])
        if other not in IN_PLACE and out not in IN_PLACE:
            assert fork(lib, **{**IN_PLACE, out: place}) == pcb.E_INVAL


@pytest.mark.parametrize("name", [*INPUTS, *OUTPUTS])
def test_arrays_in_the_workspace_are_refused(lib, name):     # noqa: F811
    assert fork(lib, **{name: WS}) == pcb.E_INVAL and fork(lib, **{name: WS + pcb.OPS_WORKSPACE_BYTES - 4}) == pcb.E_INVAL
    assert fork(lib, **{name: WS + pcb.OPS_WORKSPACE_BYTES}) == pcb.E_CUDA


@pytest.mark.parametrize("bad", [dict(n_seqs=-1), dict(n_seqs=8193), dict(n_children=-1), dict(n_children=8193), dict(page_table=None), dict(held=None),
                                 dict(length=None), dict(page_table_stride=0), dict(page_table_stride=(1 << 22) + 1), dict(parent=None), dict(table_out=None),
                                 dict(held_out=None), dict(length_out=None), dict(table_out_stride=0), dict(n_pages=0), dict(n_pages=(1 << 26) + 1), dict(refs=None),
                                 dict(free_list=None), dict(free_count=None), dict(missing=None), dict(room=-1), dict(room=(1 << 26) + 1), dict(n_pools=9), dict(n_pools=1),
                                 dict(n_pools=-1), dict(ws=None), dict(ws=WS + 128)])
def test_bad_forks_of_arrays_apart_are_refused(lib, bad):    # noqa: F811
    assert fork(lib, **bad) == pcb.E_INVAL


# ---------------------------------------------------------------------------------------------------------------- append
ROWS, HQ, HKV, D = 5, 16, 8, 128
WIDE = (HQ + 2 * HKV) * D                            # elements of a row of the projection's output
Q, K, V = A, A + 2 * HQ * D, A + 2 * (HQ + HKV) * D
APART = A + (1 << 20)


def append(lib, eight, pool=None, **kw):              # noqa: F811
    r = dict(n_seqs=2, n_rows=ROWS, max_len=128, n_q_heads=HQ, ctx_len=A + (2 << 20), row_start=A + (2 << 20) + 64, q=Q, q_out=APART, k=K, v=V, q_row_stride=WIDE,
             q_out_row_stride=HQ * D, k_row_stride=WIDE, v_row_stride=WIDE, eps=1e-6, rope=A + (3 << 20), n_positions=128)
    s = pcb.NewRowsStruct()
    for name, x in {**r, **kw}.items():
        setattr(s, name, x)
    if eight:
        kv = dict(pages=A + (4 << 20), scales=A + (5 << 20), page_stride=HKV * 32 * D, n_pages=10, page_table=A + (6 << 20), page_table_stride=8, n_kv_heads=HKV,
                  head_dim=D, dtype=0)
        p = pcb.Kv8Struct()
    else:
        kv = dict(k=A + (4 << 20), v=A + (5 << 20), k_slot_stride=HKV * D, v_slot_stride=HKV * D, n_slots=160, page_table=A + (6 << 20), page_table_stride=8, n_kv_heads=HKV,
                  head_dim=D, dtype=0)
        p = pcb.KvStruct()
    for name, x in {**kv, **(pool or {})}.items():
        setattr(p, name, x)
    return (lib.percache_append_rows_8bit if eight else lib.percache_append_rows)(NO_DEVICE, None, p, s)


@pytest.mark.parametrize("eight", [False, True])
def test_queries_go_apart_or_in_place(lib, eight):           # noqa: F811
    assert append(lib, eight) == pcb.E_CUDA
    assert append(lib, eight, q_out=Q, q_out_row_stride=WIDE) == pcb.E_CUDA                           # in place, beside k and v
    # one behind the other; a free part of the projection's rows; no queries: q_out is not looked at
    assert append(lib, eight, q_out=A + 2 * ROWS * WIDE) == pcb.E_CUDA and append(lib, eight, q_out=A - 2 * ROWS * HQ * D) == pcb.E_CUDA
    more = dict(q_row_stride=WIDE + HQ * D, k_row_stride=WIDE + HQ * D, v_row_stride=WIDE + HQ * D, q_out_row_stride=WIDE + HQ * D)
    assert append(lib, eight, q_out=A + 2 * WIDE, **more) == pcb.E_CUDA
    assert append(lib, eight, q=None, q_out=K) == pcb.E_CUDA


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("bad", [dict(q_out=K, q_out_row_stride=WIDE), dict(q_out=V, q_out_row_stride=WIDE), dict(q_out=Q + 16, q_out_row_stride=WIDE),
                                 dict(q_out=V - 16, q_out_row_stride=WIDE), dict(q_out=Q), dict(q_out=Q, q_out_row_stride=2 * WIDE), dict(q_out=K), dict(q_out=V),
                                 dict(q_out=K + 2 * WIDE, q_out_row_stride=WIDE), dict(q_out=A + 2 * ROWS * WIDE - 2 * HKV * D - 16, q_out_row_stride=HQ * D),
                                 dict(q_out=A - 2 * ROWS * HQ * D + 16), dict(q=APART, k=APART, k_row_stride=HQ * D), dict(q=A + (8 << 20), v=APART + 2 * HQ * D * 4)])
def test_queries_that_overlap_what_is_read_are_refused(lib, eight, bad):         # noqa: F811
    assert append(lib, eight, **bad) == pcb.E_INVAL


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("bad", [dict(n_seqs=-1), dict(n_seqs=65536), dict(n_rows=-1), dict(max_len=0), dict(max_len=(1 << 26) + 1), dict(ctx_len=None),
                                 dict(row_start=None), dict(k=None), dict(v=None), dict(k=K + 8), dict(v=V + 2), dict(q=Q + 8), dict(q_out=None), dict(q_out=APART + 8),
                                 dict(n_q_heads=0), dict(n_q_heads=4097), dict(q_row_stride=WIDE - 4), dict(q_row_stride=1024), dict(k_row_stride=1016),
                                 dict(v_row_stride=1020), dict(q_out_row_stride=-2048), dict(q_gain=A + 4), dict(k_gain=A + 8), dict(rope=A + 8),
                                 dict(n_positions=0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))])
def test_bad_new_rows_apart_are_refused(lib, eight, bad):    # noqa: F811
    assert append(lib, eight, **bad) == pcb.E_INVAL


@pytest.mark.parametrize("eight, bad", [(True, dict(pages=None)), (True, dict(pages=A + 8)), (True, dict(scales=None)), (True, dict(scales=A + 4)), (True, dict(page_stride=HKV * 32 * D + 16)),
                                        (True, dict(page_stride=7 * 32 * D)), (True, dict(page_stride=0)), (True, dict(n_pages=0)), (True, dict(n_pages=(1 << 26) + 1)),
                                        (True, dict(page_table=None)), (True, dict(page_table_stride=7)), (True, dict(head_dim=96)), (True, dict(dtype=2)),
                                        (False, dict(k=None)), (False, dict(v=None)), (False, dict(k_slot_stride=1020)), (False, dict(n_slots=161)),
                                        (False, dict(page_table_stride=7)), (False, dict(page_table=None)), (False, dict(head_dim=96))])
def test_bad_pools_of_rows_apart_are_refused(lib, eight, bad):       # noqa: F811
    assert append(lib, eight, pool=bad) == pcb.E_INVAL
