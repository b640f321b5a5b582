"""Attention over 8-bit pages: weights far below the row's heaviest, or below a page of a much larger scale, that are all the result is made of.

Tolerances.  A weight times its page's scale is split into parts that leave at most 2^-11 (bf16) or 2^-15 (fp16) of it, or 2^-32 or 2^-36 of the row's
largest where that is more; scores as in the other tests of this operator (Batch.delta); sums, exponentials and the division together 2^-16; the
output is rounded once.  Nothing here goes by the heavy slot's values, which are zeros where the result is looked at.
"""
import numpy as np
import pytest

from oracle import cache_ops as ops

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests.test_gpu_r_pages import TYPES, Batch, f64      # noqa: E402

KEEP = {"bf16": 2.0 ** -11, "f16": 2.0 ** -15}
FLOOR = {"bf16": 2.0 ** -32, "f16": 2.0 ** -36}
E4M3 = {0.0: 0x00, 0.05859375: 0x17, 0.1875: 0x24, 0.203125: 0x25, 0.21875: 0x26, 10.0: 0x52, 11.0: 0x53, 12.0: 0x54, 13.0: 0x55, 14.0: 0x56}


class Flat(Batch):
    """Rows of ones; a slot's score is the number that its key repeats; values positive, so that they add up."""

    def __init__(self, seqs, dtype, d=128, others=0.0, mask=None, hq=4):
        super().__init__(seqs, dtype=dtype, hq=hq, hkv=1, d=d, mask="random" if mask is not None else None)
        self.dtype = dtype
        self.q.fill_(1.0)
        self.scale = 1.0 / d
        b = self.pages.view(torch.uint8)
        own = torch.from_numpy(self.table[self.table < len(b)].astype(np.int64)).cuda()
        b[own, :, 0] = E4M3[others]
        b[own, :, 1] &= 0x3f                                   # positive, below 2
        b[own, :, 1] |= 0x20
        self.scales[:, :, 0] = 1.0
        self.scales[:, :, 1] = 2.0 ** -7
        if mask is not None:
            self.node_mask[0] = np.array(mask, dtype=bool)
            bits = np.zeros((self.n_rows, 1), dtype=np.uint64)
            for i, row in enumerate(mask):
                bits[i, 0] = sum(1 << j for j, x in enumerate(row) if x)
            self.mask = torch.from_numpy(bits.view(np.int64)).cuda()

    def slot(self, s, which):
        return self.pages.view(torch.uint8)[int(self.table[0, s // 16]), 0, which, s % 16]

    def rows_are_right(self, rows, columns, floor_from):
        """floor_from [rows]: the largest weight (of all, they sum to one) times its page's scale."""
        q, out, lse = f64(self.q), f64(self.out), f64(self.lse)
        c, n = self.seqs[0]
        k, v = self.kv(0, c + n)
        want, wlse, mean_abs = ops.tree_attention(q[:n], k, v, c, self.node_mask[0], self.scale)
        delta = self.delta(q[:n], k, ops.sees(n, c, self.node_mask[0]))
        eps = torch.finfo(TYPES[self.dtype]).eps / 2
        seen = ops.sees(n, c, self.node_mask[0])
        scales = np.repeat(f64(self.scales[torch.from_numpy(self.table[0, :-(-(c + n) // 16)].astype(np.int64)).cuda()])[:, 0, 1], 16)[:c + n]
        for r in rows:
            # what the floor may take from every slot: its bytes times that
            raw = np.abs(v[:, 0] / scales[:, None])[seen[r]][:, columns].sum(0)
            # half a step of the output: eps of the value, and below 2^-14 fp16's steps are 2^-24 (its subnormal numbers), bf16's never that coarse
            half_step = np.maximum(eps * np.abs(want[r]), 2.0 ** -25 if self.dtype == "f16" else 0.0)
            tol = half_step + (KEEP[self.dtype] + 2 * delta[r][:, None] + 2.0 ** -16) * mean_abs[r]
            tol = tol[:, columns] + FLOOR[self.dtype] * floor_from[r] * raw
            # the floor must not be what lets a wrong result through
            assert (tol <= 2.0 ** -6 * np.abs(want[r][:, columns])).all()
            diff = np.abs(out[r] - want[r])[:, columns]
            assert (diff <= tol).all(), (r, (diff / np.abs(want[r][:, columns])).max(), (diff / tol).max())
            assert (np.abs(lse[r] - wlse[r]) <= delta[r] + 2.0 ** -20 * (np.abs(wlse[r]) + 4)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d, hq", [(128, 4), (64, 4), (128, 24)])
@pytest.mark.parametrize("heavy", [10.0, 11.0, 12.0, 13.0, 14.0])
@pytest.mark.parametrize("others", [0.0, 0.1875, 0.21875])
def test_many_equal_slots_under_a_heavy_one(dtype, d, hq, heavy, others):
    """2000 slots of one weight, 2^-14 to 2^-20 of a slot whose value is zero: their common rounding is the result's."""
    b = Flat([(2000, 1)], dtype, d=d, others=others, hq=hq)
    b.slot(5, 0)[:] = E4M3[heavy]
    b.slot(5, 1)[:] = 0
    b.attend()
    b.rows_are_right([0], np.arange(d), [2.0 ** -7])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("but_one", [False, True])
@pytest.mark.parametrize("up", [3, 8, 12, 15, 18, 20, 22])
def test_a_page_of_a_larger_scale_does_not_hide_the_others(dtype, but_one, up):
    """A page whose values' scale is 2^up times the others', its bytes zeros in all elements or in all but one."""
    b = Flat([(900, 2)], dtype, others=0.05859375)
    page = int(b.table[0, 7])
    b.pages.view(torch.uint8)[page, 0, 0] = E4M3[0.0]
    b.pages.view(torch.uint8)[page, 0, 1] = 0
    if but_one:
        b.pages.view(torch.uint8)[page, 0, 1, :, 77] = 0x7e
    b.scales[page, 0, 1] = 2.0 ** (up - 7)
    b.attend()
    b.rows_are_right([0, 1], np.delete(np.arange(128), 77), [2.0 ** (up - 7) / 800] * 2)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("up", [8, 13, 16, 20])
def test_an_outlier_in_a_drafted_sibling_does_not_hide_what_others_see(dtype, up):
    """Node 3's value sets the scale of a page that it shares with slots that rows 0 to 2 see, whose bytes are zeros beside it; no row but its own sees it."""
    mask = [[1, 0, 0, 0], [1, 1, 0, 0], [1, 0, 1, 0], [1, 0, 0, 1]]
    b = Flat([(405, 4)], dtype, others=0.05859375, mask=mask)
    page = int(b.table[0, 408 // 16])
    b.pages.view(torch.uint8)[page, 0, 0] = E4M3[0.0]
    b.pages.view(torch.uint8)[page, 0, 1] = 0
    b.slot(408, 1)[:] = 0x7e
    b.scales[page, 0, 1] = 2.0 ** (up - 7)
    b.attend()
    b.rows_are_right([0, 1, 2], np.arange(128), [2.0 ** (up - 7) / 390] * 3)
    assert np.isfinite(f64(b.out[3])).all() and (f64(b.out[3]) > 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("seqs, hq", [([(700, 1)] * 8, 4), ([(700, 9)] * 2, 8)])
def test_the_error_is_the_last_roundings(dtype, seqs, hq):
    """Weights off by 2^-12 (bf16) or 2^-16 (fp16) of themselves, independent of each other, are off by that much of the result: beside the output's own
    rounding (2^-9.2 and 2^-12.2 on average) their square adds less than a twentieth."""
    b = Batch(seqs, dtype=dtype, hq=hq, hkv=2, q_scale=0.3)
    b.attend()
    out = b.out.double().cpu()
    got = rounded = 0.0
    for i, (c, n) in enumerate(seqs):
        r = slice(int(b.row_start[i]), int(b.row_start[i + 1]))
        k, v = b.kv(i, c + n)
        want = torch.from_numpy(ops.tree_attention(f64(b.q[r]), k, v, c, None, b.scale)[0])
        got += float(((out[r] - want) ** 2).sum())
        rounded += float(((want.to(TYPES[dtype]).double() - want) ** 2).sum())
    assert got <= 1.05 ** 2 * rounded, (got / rounded) ** 0.5
