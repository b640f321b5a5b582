"""Refusals of the cache operators that used to come late or not at all.  None needs a device."""
from paper_2601_11553_b200 import percache as pcb
from tests.test_ops_abi import compact, kv, lib                        # noqa: F401


def test_more_heads_than_a_grid_has_rows_cannot_be_moved(lib):                      # noqa: F811
    wide = kv(n_kv_heads=65536, head_dim=64, k_slot_stride=65536 * 64, v_slot_stride=65536 * 64)
    assert compact(lib, wide, heads=1) == pcb.E_INVAL
