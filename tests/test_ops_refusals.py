"""Refusals of the cache operators that used to come late or not at all.  None needs a device."""
import pytest

from paper_2601_11553_b200 import percache as pcb
from tests.test_ops_abi import A, compact, kv, lib, rows, tree, weights       # noqa: F401


def test_more_heads_than_a_grid_has_rows_cannot_be_moved(lib):                      # noqa: F811
    wide = kv(n_kv_heads=65536, head_dim=64, k_slot_stride=65536 * 64, v_slot_stride=65536 * 64)
    assert compact(lib, wide, heads=1) == pcb.E_INVAL


def test_weights_out_without_weights_is_refused():
    torch = pytest.importorskip("torch")
    k = torch.zeros((16, 2, 128), dtype=torch.float16)
    with pytest.raises(ValueError, match="weights_out"):
        pcb.compact_slots(k, k, torch.zeros((1, 2, 4), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), max_len=16,
                          weights_out=torch.zeros((1, 2, 16)), ctx_start=torch.zeros(1, dtype=torch.int32))


def test_more_work_than_the_schedule_counts_is_refused_before_a_device_is_looked_for(lib):    # noqa: F811
    long = kv(page_table=None, ctx_start=A)
    batch = rows(n_seqs=65535, n_rows=65535, max_nodes=1, max_len=1 << 26)
    assert tree(lib, long, batch) == pcb.E_CAPACITY
    assert weights(lib, long, batch, stride=1 << 26) == pcb.E_CAPACITY
    many = kv(page_table=None, ctx_start=A, n_kv_heads=4096, k_slot_stride=4096 * 128, v_slot_stride=4096 * 128)
    batch = rows(n_seqs=1, max_nodes=256, max_len=1 << 26)
    assert tree(lib, many, batch, hq=4096 * 128, q_stride=4096 * 128 * 128, out_stride=4096 * 128 * 128) == pcb.E_CAPACITY
