"""Pins of the oracle of the operators on pages: hand-worked cases and an independent cast."""
import numpy as np
import pytest

from oracle import pages as P


def test_bytes_stand_for_what_the_format_says():
    assert P.VALUES[0x7e] == 448 and P.VALUES[0x01] == 2.0 ** -9 and P.VALUES[0x08] == 2.0 ** -6 and P.VALUES[0x38] == 1.0 and P.VALUES[0xb8] == -1.0
    assert np.isnan(P.VALUES[0x7f]) and np.isnan(P.VALUES[0xff])


def test_rounding_agrees_with_a_library_cast():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(20000) * 2.0 ** rng.integers(-12, 9, 20000), (P.VALUES[:126] + P.VALUES[1:127]) / 2, P.VALUES[:127]])
    x = np.concatenate([x, -x]).astype(np.float32)
    x = x[np.abs(x) <= 448]
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(P.to_e4m3(x), want)


def test_large_values_saturate_and_nan_stays():
    assert list(P.to_e4m3([1e9, -1e9, np.inf, -np.inf, 464.0])) == [0x7e, 0xfe, 0x7e, 0xfe, 0x7e]
    assert P.to_e4m3([np.nan])[0] & 0x7f == 0x7f


@pytest.mark.parametrize("amax, e", [(0.0, -32), (448.0, 0), (448.0000001, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.76, -7), (1e30, 32)])
def test_scales(amax, e):
    assert P.scale_exponent(amax) == e


def test_a_page_that_grows_keeps_its_values():
    raw, s = np.zeros((16, 4), dtype=np.uint8), 123.0                       # an unused page's scale means nothing
    raw, s = P.fill_page(raw, s, 0, np.full((3, 4), 1.5))
    assert s == 2.0 ** -8 and (P.VALUES[raw[:3]] * s == 1.5).all()
    raw, s = P.fill_page(raw, s, 3, np.full((1, 4), -7.0))
    assert s == 2.0 ** -6 and (P.VALUES[raw[:3]] * s == 1.5).all() and (P.VALUES[raw[3]] * s == -7).all()
    again, s2 = P.fill_page(raw, s, 4, np.full((1, 4), 0.25))
    assert s2 == s and np.array_equal(again[:4], raw[:4]) and (P.VALUES[again[4]] * s == 0.25).all()


def test_fork_by_hand():
    # sequence 0: pages 5, 2, 7 with 40 slots (page 7 half full); sequence 1: pages 5, 9 with 20; sequence 2: page 4, empty
    table = [[5, 2, 7], [5, 9, -1], [4, -1, -1]]
    refs = [0, 0, 1, 0, 1, 2, 0, 1, 0, 1, 0]
    out, held, length, refs, free, missing, copies = P.fork(table, [3, 2, 1], [40, 20, 0], [0, 0, 2, 0], 4, refs, [10, 8, 6, 3, 1], 8, 11)
    # room for 8 more: 48 slots, three pages.  Child 0 goes on with 5, 2, 7; child 1 copies 7 to 1, child 3 to 3; child 2 keeps 4
    assert out == [[5, 2, 7], [5, 2, 1], [4], [5, 2, 3]]
    assert held == [3, 3, 1, 3] and length == [40, 40, 0, 40] and missing == 0 and copies == [(7, 1), (7, 3)]
    assert refs == [0, 1, 3, 1, 1, 3, 0, 1, 0, 0, 0] and free == [10, 8, 6, 9]          # sequence 1 let go of 5 (held on) and 9


def test_fork_gives_everything_back_and_says_what_is_missing():
    out, held, length, refs, free, missing, copies = P.fork([[1, 0]], [2], [32], [], 2, [1, 1, 0], [2], 0, 3)
    assert out == [] and refs == [0, 0, 0] and free == [2, 0, 1]
    out, held, length, refs, free, missing, copies = P.fork([[1, 0]], [2], [20], [0, 0, 0], 2, [1, 1, 0], [2], 0, 3)
    assert out == [[1, 0], [1, 2], [1]] and length == [20, 20, 16] and missing == 1 and copies == [(0, 2)] and refs == [1, 3, 1]
