"""Refusals of the cache operators: every one is decided on the host, before a device is looked for."""
import ctypes as C

import pytest

from paper_2601_11553_b200 import percache as pcb

A = 1 << 20          # an address that is never followed: these calls are refused before anything runs


@pytest.fixture(scope="module")
def lib():
    from paper_2601_11553_b200 import build
    build.build()
    return pcb.load_library()


def kv(**kw):
    s = pcb.KvStruct(A, A, 1024, 1024, 160, A, None, 8, 8, 128, 0)
    for k, x in kw.items():
        setattr(s, k, x)
    return s


def rows(**kw):
    s = pcb.RowsStruct(2, 3, 2, 128, A, A, None, 0, 0)
    for k, x in kw.items():
        setattr(s, k, x)
    return s


def tree(lib, kvs=None, rs=None, q=A, q_stride=2048, hq=16, scale=0.1, out=A, out_stride=2048, lse=A, ws=A, nbytes=24 << 20, device=0):
    return lib.percache_tree_attention(device, None, kvs or kv(), rs or rows(), q, q_stride, hq, scale, out, out_stride, lse, ws, nbytes)


def weights(lib, kvs=None, rs=None, q=A, q_stride=2048, hq=16, scale=0.1, lse=A, use=None, decay=1.0, w_in=A, w_out=A, stride=128,
            ws=A, nbytes=24 << 20):
    return lib.percache_attention_weights(0, None, kvs or kv(), rs or rows(), q, q_stride, hq, scale, lse, use, decay, w_in, w_out,
                                          stride, ws, nbytes)


def select(lib, w=A, stride=128, length=A, n=2, heads=8, max_len=128, budget=16, sink=4, recent=8, keep=A, count=A):
    return lib.percache_select_slots(0, None, w, stride, length, n, heads, max_len, budget, sink, recent, keep, count)


def compact(lib, kvs=None, n=2, max_len=128, dpt=None, dpt_stride=0, dst=None, first=None, keep=A, heads=8, budget=16, count=A,
            w_in=None, w_out=None, stride=0):
    return lib.percache_compact_slots(0, None, kvs or kv(), n, max_len, dpt, dpt_stride, dst, first, keep, heads, budget, count,
                                      w_in, w_out, stride)


BAD_KV = [dict(k=None), dict(k=A + 8), dict(k_slot_stride=1020), dict(k_slot_stride=512), dict(n_slots=0), dict(n_slots=1 << 31),
          dict(n_slots=161), dict(page_table_stride=7), dict(page_table=None), dict(n_kv_heads=0), dict(head_dim=96), dict(dtype=2)]


@pytest.mark.parametrize("bad", BAD_KV)
def test_bad_pools_are_refused(lib, bad):
    assert tree(lib, kv(**bad)) == pcb.E_INVAL
    assert weights(lib, kv(**bad)) == pcb.E_INVAL
    assert compact(lib, kv(**bad)) == pcb.E_INVAL


@pytest.mark.parametrize("bad", [dict(v=None), dict(v=A + 4), dict(v_slot_stride=1000), dict(v_slot_stride=8)])
def test_bad_values_are_refused(lib, bad):
    assert tree(lib, kv(**bad)) == pcb.E_INVAL
    assert compact(lib, kv(**bad)) == pcb.E_INVAL


@pytest.mark.parametrize("bad", [dict(n_seqs=-1), dict(n_rows=-1), dict(max_nodes=0), dict(max_nodes=257), dict(max_len=0),
                                 dict(ctx_len=None), dict(row_start=None), dict(mask=A, mask_words=0),
                                 dict(max_nodes=65, mask=A, mask_words=1), dict(max_len=(1 << 26) + 1), dict(n_seqs=65536)])
def test_bad_rows_are_refused(lib, bad):
    assert tree(lib, rs=rows(**bad)) == pcb.E_INVAL
    assert weights(lib, rs=rows(**bad)) == pcb.E_INVAL


def test_bad_arguments_of_tree_attention(lib):
    for bad in (dict(q=None), dict(q=A + 2), dict(q_stride=2044), dict(q_stride=1024), dict(hq=12), dict(hq=0), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(out=None), dict(out=A + 8),
                dict(out_stride=2047), dict(out_stride=2040), dict(ws=None), dict(ws=A + 128), dict(hq=8 * 129, q_stride=132096, out_stride=132096)):
        assert tree(lib, **bad) == pcb.E_INVAL, bad
    assert tree(lib, nbytes=(24 << 20) - 1) == pcb.E_CAPACITY


def test_bad_arguments_of_attention_weights(lib):
    for bad in (dict(q=None), dict(lse=None), dict(decay=-1.0), dict(decay=float("nan")), dict(w_in=None), dict(w_out=None),
                dict(stride=127), dict(ws=None), dict(hq=9)):
        assert weights(lib, **bad) == pcb.E_INVAL, bad
    assert weights(lib, nbytes=1024) == pcb.E_CAPACITY
    assert weights(lib, rs=rows(n_rows=0), hq=8 * 129) == pcb.E_INVAL          # also where there is no row to look at


def test_bad_arguments_of_select_and_compact(lib):
    for bad in (dict(w=None), dict(stride=100), dict(length=None), dict(n=-1), dict(heads=0), dict(max_len=0), dict(budget=0),
                dict(sink=-1), dict(recent=-1), dict(sink=9), dict(keep=None), dict(count=None), dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1)):
        assert select(lib, **bad) == pcb.E_INVAL, bad
    assert select(lib, budget=(1 << 26) + 1) == pcb.E_INVAL
    for bad in (dict(keep=None), dict(count=None), dict(heads=2), dict(budget=0), dict(dst=A), dict(dpt=A, dst=A), dict(dpt=A, dpt_stride=0),
                dict(w_in=A), dict(w_out=A), dict(w_in=A, w_out=A, stride=127), dict(max_len=0), dict(n=-1),
                dict(kvs=kv(page_table=None, ctx_start=A), dpt=A, dpt_stride=8)):
        assert compact(lib, **bad) == pcb.E_INVAL, bad


def test_an_empty_batch_is_no_error_and_needs_no_device(lib):
    assert tree(lib, rs=rows(n_seqs=0)) == pcb.OK
    assert tree(lib, rs=rows(n_rows=0)) == pcb.OK
    assert weights(lib, rs=rows(n_seqs=0)) == pcb.OK
    assert select(lib, n=0) == pcb.OK
    assert compact(lib, n=0) == pcb.OK


def test_no_device_is_an_error_and_not_a_fallback(lib):
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert tree(lib) == pcb.E_CUDA
    assert weights(lib) == pcb.E_CUDA
    assert select(lib) == pcb.E_CUDA
    assert compact(lib) == pcb.E_CUDA
    assert lib.percache_ops_status(0, None, A) == pcb.E_CUDA
    assert lib.percache_ops_status(0, None, None) == pcb.E_INVAL


def test_struct_sizes_match_the_header():
    assert C.sizeof(pcb.KvStruct) == 72
    assert C.sizeof(pcb.RowsStruct) == 48


def test_binding_refuses_tensors_it_cannot_pass_on():
    torch = pytest.importorskip("torch")
    k = torch.zeros((16, 2, 128), dtype=torch.float16)
    with pytest.raises(ValueError):                      # host memory
        pcb.compact_slots(k, k, torch.zeros((1, 2, 4), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), max_len=16,
                          ctx_start=torch.zeros(1, dtype=torch.int32))
