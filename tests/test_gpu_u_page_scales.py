"""New rows into 8-bit pages whose scale is no power of two (pages that something else wrote): bytes are x / scale rounded once, bit for bit.

A product with the reciprocal, and a quotient in fp32 too, are rounded before the rounding to 8 bits: next to the border of two bytes that can be the other one.
"""
import numpy as np
import pytest

from oracle import pages as P

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests.test_gpu_r_pages import Rows, raw      # noqa: E402

BORDERS = (P.VALUES[:118] + P.VALUES[1:119]) / 2      # below 224: times a scale below 448 times the power of two under it, which keeps the scale
# few rows: by the kernel that has a page a warp; many: by the one of long prompts; 2**18 heads of rows and 64 rows a prompt are its border
FEW, MANY = [(5 + 3 * i % 11, 1 + i % 5) for i in range(20)], [(3 + 5 * i % 13, 66) for i in range(1000)]


def first_pages(r):
    return torch.from_numpy(np.array([r.table[b, c // 16] for b, (c, _) in enumerate(r.seqs)]).astype(np.int64)).cuda()


def scales_of(r, values):
    """One of the values for every prompt's first page."""
    s = np.array(values, dtype=np.float32)[np.arange(len(r.seqs)) % len(values)]
    r.scales[first_pages(r)] = torch.from_numpy(s).cuda()[:, None, None]
    return s


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("seqs", [FEW, MANY], ids=["few", "many"])
def test_values_at_the_borders_of_a_kept_scale(dtype, d, seqs):
    """The page's scale stays: values at the borders of two bytes times the scale, as near as the type has them, are rounded as their quotient is."""
    r = Rows(seqs, dtype=dtype, hkv=2, d=d, norm=False, rope=False)
    rng = np.random.default_rng(0)
    s = scales_of(r, [7 * 2.0 ** -9, 1.3 * 2.0 ** -8, 1.1 * 2.0 ** -8, 3 * 2.0 ** -9, *(rng.uniform(1, 2, 5) * 2.0 ** -8)])
    rows = np.repeat(s.astype(np.float64), [n for _, n in seqs])
    for x in (r.k, r.v):
        at = rng.choice(BORDERS, (r.n, 2, d)) * rng.choice([-1.0, 1.0], (r.n, 2, d))
        x[:r.n] = torch.from_numpy(at * rows[:, None, None]).cuda().to(x.dtype)
    r.before = raw(r.pages).copy(), r.scales.cpu().numpy().copy()
    r.run(q=False)
    r.check(q=False)
    assert torch.equal(r.scales[first_pages(r)].cpu(), torch.from_numpy(s)[:, None, None].expand(len(s), 2, 2))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("seqs", [FEW, MANY], ids=["few", "many"])
def test_bytes_that_are_rounded_again_from_such_a_scale(d, seqs):
    """The scale grows to a power of two: every byte there is times a factor that is none."""
    r = Rows(seqs, hkv=2, d=d, norm=False, rope=False)
    near = [np.nextafter(np.float32(a / b), np.float32(to)) for a, b in ((17, 18), (19, 18), (21, 20), (27, 26), (17, 20), (29, 24)) for to in (0, 2)]
    scales_of(r, [np.float32(2.0 ** -12) * x for x in near + [np.float32(17 / 18), np.float32(19 / 18), np.float32(27 / 26), np.float32(1.1), np.float32(1.7)]])
    r.pages.view(torch.uint8)[first_pages(r)] = torch.randint(0, 256, (len(seqs), 2, 2, 16, d), device="cuda", dtype=torch.uint8,
                                                                generator=torch.Generator(device="cuda").manual_seed(1))
    r.before = raw(r.pages).copy(), r.scales.cpu().numpy().copy()
    r.run(q=False)
    now = r.scales[first_pages(r)].cpu().numpy()
    assert (np.frexp(now)[0] == 0.5).all() and (now > 2.0 ** -11).any()
    nan = (raw(r.pages) & 0x7f) == 0x7f
    assert np.array_equal(nan[first_pages(r).cpu().numpy()][:, :, :, 0], (r.before[0][first_pages(r).cpu().numpy()][:, :, :, 0] & 0x7f) == 0x7f)
    r.check(q=False)


def test_infinities_and_nan_beside_such_a_scale():
    r = Rows([(3, 5)], hkv=2, norm=False, rope=False)
    scales_of(r, [7 * 2.0 ** -9])
    r.k[:5], r.v[:5] = r.k[:5].clamp(-4, 4), r.v[:5].clamp(-4, 4)
    r.k[0, 0, 3], r.k[1, 0, 5], r.k[2, 1, 7], r.v[3, 1, 9] = float("inf"), float("-inf"), float("nan"), 1e-30
    r.before = raw(r.pages).copy(), r.scales.cpu().numpy().copy()
    r.run(q=False)
    k = raw(r.pages)[r.table[0, 0]][:, 0]
    assert k[0, 3, 3] == 0x7e and k[0, 4, 5] == 0xfe and k[1, 5, 7] & 0x7f == 0x7f
    assert raw(r.pages)[r.table[0, 0]][1, 1, 6, 9] == 0
