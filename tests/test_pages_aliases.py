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
