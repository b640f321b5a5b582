"""Forks on both sides of the sizes up to which one kernel does them."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests.test_gpu_r_pages import Forest      # noqa: E402

BORDERS = [
    # (sequences, slots of each, children, table width, pages)
    (128, 20, 128, 10, 2000), (129, 20, 129, 10, 2000), (128, 20, 512, 10, 2000), (128, 20, 513, 10, 2000), (128, 100, 100, 80, 4096), (128, 100, 100, 81, 4096),
    (3, 700, 40, 60, 4096), (3, 700, 40, 60, 4097), (1, 37, 512, 8, 4096), (1, 37, 513, 8, 4097),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n, slots, children, width, pages", BORDERS)
def test_forks_around_the_border(n, slots, children, width, pages, in_place):
    lengths = [max(1, slots - i % 23) for i in range(n)]
    used = 1 + sum(-(-x // 16) - 1 for x in lengths)
    f = Forest(lengths, shared=1, spare=pages - used, width=width, layers=1, pool_kinds=("f8", "scale"), seed=n)
    assert f.total == pages
    f.fork([(i * i + i // 3) % n if i % 17 else -1 for i in range(children)], room=5, in_place=in_place)
    f.fork(list(range(0, children, 2))[:n], room=0, in_place=in_place)
