"""Batches most of whose prompts have no rows: runs of them between, ahead of and behind the others."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests import test_gpu_m_cache_ops as M      # noqa: E402
from tests.test_gpu_r_pages import Batch, Rows      # noqa: E402

RUNS = [1, 31, 32, 33, 64, 127, 128, 250, 1000]


def between(work, idle, run):
    """Idle prompts in runs ahead of, between and behind the working ones; one run is twice as long."""
    seqs = [idle] * run
    for i, w in enumerate(work):
        seqs += [w] + [idle] * (run * 2 if i == 0 else run)
    return seqs


@pytest.mark.parametrize("run", RUNS)
@pytest.mark.parametrize("cache", ["8bit", "pages", "slots"])
@pytest.mark.parametrize("idle", [(0, 0), (37, 0)])
def test_new_rows_of_few_prompts(run, cache, idle):
    r = Rows(between([(5, 203), (0, 1), (16, 40), (3, 5)], idle, run), cache=cache)
    r.run()
    r.check()


@pytest.mark.parametrize("run", [40, 130])
@pytest.mark.parametrize("cache", ["8bit", "pages"])
def test_many_new_rows_of_few_prompts(run, cache):
    """Enough rows a prompt on average for the kernel of long prompts."""
    n = 64 * (4 * run + 3) if cache == "8bit" else 16 * (4 * run + 3)
    n = max(n, 9000)
    r = Rows(between([(5, n // 2 + 7), (16, 3), (9, n // 2 + 301)], (20, 0), run), cache=cache, hq=16, hkv=8)
    r.run()
    r.check()


@pytest.mark.parametrize("run", RUNS)
@pytest.mark.parametrize("kw", [dict(hq=4, hkv=2), dict(hq=16, hkv=2, dtype="f16", mask="tree"), dict(hq=4, hkv=1, d=64)])
def test_attention_over_8_bit_pages_of_few_prompts(run, kw):
    b = Batch(between([(900, 3), (0, 1), (130, 9), (2000, 1), (60, 2)], (0, 0) if run % 2 else (37, 0), run), **kw)
    b.attend()
    b.check()


@pytest.mark.parametrize("run", RUNS)
@pytest.mark.parametrize("kw", [dict(hq=4, hkv=2), dict(hq=16, hkv=2, dtype="f16", mask="tree"), dict(hq=8, hkv=1, paged=False)])
def test_attention_over_16_bit_slots_of_few_prompts(run, kw):
    b = M.Batch(between([(900, 3), (0, 1), (130, 9), (2000, 1), (60, 2)], (0, 0) if run % 2 else (37, 0), run), **kw)
    b.attend()
    b.check()


@pytest.mark.parametrize("run", RUNS)
@pytest.mark.parametrize("kw", [dict(hq=4, hkv=2), dict(hq=16, hkv=2, dtype="f16", mask="tree")])
def test_attention_weights_of_few_prompts(run, kw):
    b = M.Batch(between([(900, 3), (0, 1), (130, 9), (60, 2)], (0, 0), run), **kw)
    b.attend()
    w = torch.rand((len(b.seqs), b.hkv, b.max_len), device="cuda")
    before = w.clone()
    M.pcb.attention_weights(b.q, b.k, b.lse, w, **b.args())
    M.check_weights(b, w, before, None, 1.0)
