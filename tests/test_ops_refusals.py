"""Refusals of the cache operators that used to come late or not at all.  None needs a device."""
import pytest

from paper_2601_11553_b200 import percache as pcb
from tests.test_ops_abi import compact, kv, lib                        # noqa: F401


def test_more_heads_than_a_grid_has_rows_cannot_be_moved(lib):                      # noqa: F811
    wide = kv(n_kv_heads=65536, head_dim=64, k_slot_stride=65536 * 64, v_slot_stride=65536 * 64)
    assert compact(lib, wide, heads=1) == pcb.E_INVAL


def test_weights_out_without_weights_is_refused():
    torch = pytest.importorskip("torch")
    k = torch.zeros((16, 2, 128), dtype=torch.float16)
    with pytest.raises(ValueError, match="weights_out"):
        pcb.compact_slots(k, k, torch.zeros((1, 2, 4), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), max_len=16,
                          weights_out=torch.zeros((1, 2, 16)), ctx_start=torch.zeros(1, dtype=torch.int32))
