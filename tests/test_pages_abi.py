"""Refusals of the operators on pages: decided on the host, before a device is looked for."""
import ctypes as C

import pytest

from paper_2601_11553_b200 import percache as pcb
from tests.test_ops_abi import A, kv, lib, rows       # noqa: F401


def kv8(**kw):
    s = pcb.Kv8Struct(A, A, 8 * 32 * 128, 10, A, 8, 8, 128, 0)
    for k, x in kw.items():
        setattr(s, k, x)
    return s


def new_rows(**kw):
    s = pcb.NewRowsStruct(2, 3, 128, 16, A, A, None, A, A, A, A, 4096, 2048, 4096, 4096, A, A, A, 128, 1e-6)
    for k, x in kw.items():
        setattr(s, k, x)
    return s


def append(lib, pool=None, r=None):                   # noqa: F811
    return lib.percache_append_rows(0, None, pool or kv(), r or new_rows())


def append8(lib, pool=None, r=None):                  # noqa: F811
    return lib.percache_append_rows_8bit(0, None, pool or kv8(), r or new_rows())


def tree8(lib, pool=None, rs=None, q=A, q_stride=2048, hq=16, scale=0.1, out=A, out_stride=2048, lse=A, ws=A, nbytes=24 << 20):   # noqa: F811
    return lib.percache_tree_attention_8bit(0, None, pool or kv8(), rs or rows(), q, q_stride, hq, scale, out, out_stride, lse, ws, nbytes)


def fork(lib, ws=A, nbytes=24 << 20, pools=None, **kw):       # noqa: F811
    s = pcb.ForkStruct(2, 3, 8, 8, A, A, A, A, A + 4096, A + 4096, A + 4096, 100, A, A, A, A, A, A, A, 1, 0, None)
    if pools is not None:
        arr = (pcb.PoolStruct * len(pools))(*pools)
        s.pools, s.n_pools = C.cast(arr, C.POINTER(pcb.PoolStruct)), len(pools)
    for k, x in kw.items():
        setattr(s, k, x)
    return lib.percache_fork_pages(0, None, C.byref(s), ws, nbytes)


@pytest.mark.parametrize("bad", [dict(pages=None), dict(pages=A + 8), dict(scales=None), dict(scales=A + 4), dict(page_stride=8 * 32 * 128 + 16),
                                 dict(page_stride=7 * 32 * 128), dict(page_stride=0), dict(page_stride=-8 * 32 * 128), dict(n_pages=0),
                                 dict(n_pages=(1 << 26) + 1), dict(n_pages=1 << 26, page_stride=32 * 32 * 128), dict(page_table=None), dict(page_table_stride=7),
                                 dict(n_kv_heads=0), dict(n_kv_heads=4097), dict(head_dim=96), dict(head_dim=256), dict(dtype=2)])
def test_bad_8bit_pages_are_refused(lib, bad):               # noqa: F811
    assert tree8(lib, kv8(**bad)) == pcb.E_INVAL
    assert append8(lib, kv8(**bad)) == pcb.E_INVAL


@pytest.mark.parametrize("bad", [dict(n_seqs=-1), dict(n_seqs=65536), dict(n_rows=-1), dict(max_len=0), dict(max_len=(1 << 26) + 1), dict(ctx_len=None),
                                 dict(row_start=None), dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 2), dict(q=A + 8), dict(q_out=None), dict(q_out=A + 8),
                                 dict(n_q_heads=0), dict(n_q_heads=4097), dict(q_row_stride=2044), dict(q_row_stride=1024), dict(k_row_stride=1016),
                                 dict(v_row_stride=1020), dict(q_out_row_stride=-2048), dict(q_gain=A + 4), dict(k_gain=A + 8), dict(rope=A + 8),
                                 dict(n_positions=0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                                 dict(q_out=A, q_out_row_stride=2048)])      # in place with another stride
def test_bad_new_rows_are_refused(lib, bad):                 # noqa: F811
    assert append(lib, r=new_rows(**bad)) == pcb.E_INVAL
    assert append8(lib, r=new_rows(**bad)) == pcb.E_INVAL


def test_bad_16_bit_pools_are_refused(lib):                  # noqa: F811
    for bad in (dict(k=None), dict(v=None), dict(k_slot_stride=1020), dict(n_slots=161), dict(page_table_stride=7), dict(page_table=None), dict(head_dim=96)):
        assert append(lib, kv(**bad)) == pcb.E_INVAL


def test_empty_batches_are_fine_without_anything_else(lib):  # noqa: F811
    assert append(lib, r=new_rows(n_seqs=0, k=None)) == 0 and append8(lib, r=new_rows(n_rows=0, k=None)) == 0
    assert tree8(lib, rs=rows(n_seqs=0), q=None) == 0 and tree8(lib, rs=rows(n_rows=0), q=None) == 0


def test_bad_attention_calls_are_refused(lib):               # noqa: F811
    for bad in (dict(n_seqs=-1), dict(n_seqs=65536), dict(max_nodes=0), dict(max_nodes=257), dict(max_len=0), dict(ctx_len=None), dict(row_start=None)):
        assert tree8(lib, rs=rows(**bad)) == pcb.E_INVAL
    assert tree8(lib, rs=rows(mask=A, mask_words=0)) == pcb.E_INVAL
    for bad in (dict(q=None), dict(q=A + 2), dict(hq=12), dict(hq=0), dict(hq=8 * 129, q_stride=1 << 20, out_stride=1 << 20), dict(q_stride=1024), dict(q_stride=2052),
                dict(scale=0.0), dict(scale=float("nan")), dict(out=None), dict(out=A + 8), dict(out_stride=2044), dict(ws=None), dict(ws=A + 128)):
        assert tree8(lib, **bad) == pcb.E_INVAL, bad
    assert tree8(lib, nbytes=1 << 20) == pcb.E_CAPACITY


def test_more_work_than_the_schedule_counts_is_refused(lib):  # noqa: F811
    assert tree8(lib, kv8(page_table_stride=1 << 22), rows(n_seqs=65535, n_rows=65535, max_nodes=256, max_len=1 << 26)) == pcb.E_CAPACITY


POOL = (A, 4096, 4096, 40960, 2, 0)


@pytest.mark.parametrize("bad", [dict(n_seqs=-1), dict(n_seqs=8193), dict(n_children=-1), dict(n_children=8193), dict(page_table=None), dict(held=None),
                                 dict(length=None), dict(page_table_stride=0), dict(page_table_stride=(1 << 22) + 1), dict(parent=None), dict(table_out=None),
                                 dict(held_out=None), dict(length_out=None), dict(table_out_stride=0), dict(table_out=A), dict(held_out=A), dict(length_out=A),
                                 dict(n_pages=0), dict(n_pages=(1 << 26) + 1), dict(refs=None), dict(free_list=None), dict(free_count=None),
                                 dict(missing=None), dict(refs_out=A + 4096), dict(free_list_out=A + 4096), dict(free_count_out=A + 4096),
                                 dict(refs_out=A + 4096, free_list_out=A + 4096), dict(room=-1), dict(room=(1 << 26) + 1), dict(n_pools=9), dict(n_pools=1),
                                 dict(n_pools=-1), dict(ws=None), dict(ws=A + 128)])
def test_bad_forks_are_refused(lib, bad):                    # noqa: F811
    assert fork(lib, **bad) == pcb.E_INVAL


@pytest.mark.parametrize("at, value", [(0, None), (0, A + 2), (1, 0), (1, 4098), (2, 4092), (2, 4098), (3, 40962), (3, -4096), (4, 0), (4, 65536)])
def test_bad_pools_of_a_fork_are_refused(lib, at, value):    # noqa: F811
    pool = list(POOL)
    pool[at] = value
    assert fork(lib, pools=[pcb.PoolStruct(*POOL), pcb.PoolStruct(*pool)]) == pcb.E_INVAL


def test_a_small_workspace_is_refused(lib):                  # noqa: F811
    assert fork(lib, nbytes=1 << 20) == pcb.E_CAPACITY


def test_python_refusals():
    torch = pytest.importorskip("torch")
    k = torch.zeros((3, 2, 128), dtype=torch.float16)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        pcb.append_rows(None, k, k, ctx_len=i, row_start=i, max_len=16, k_pool=k, v_pool=k, ctx_start=i)
    with pytest.raises(ValueError, match="CUDA"):
        pcb.tree_attention_8bit(k, k, k, k, ctx_len=i, row_start=i, page_table=i, max_nodes=1, max_len=16, workspace=i)
    with pytest.raises(ValueError, match="CUDA"):
        pcb.fork_pages(i, i, i, i, i, i, i, i, i, i, i, workspace=i)
