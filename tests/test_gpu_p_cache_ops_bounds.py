"""The cache operators' dealing of work for many prompts, and device-side values beyond the bounds the host gave."""
import pytest

from paper_2601_11553_b200 import percache as pcb
from tests.test_gpu_m_cache_ops import Batch, check_weights

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("nodes,kw", [(3, dict(hq=2, hkv=1)), (3, dict(hq=4, hkv=2, dtype="f16", paged=False)), (40, dict(hq=4, hkv=1))])
def test_many_prompts_with_long_ones_among_them(nodes, kw):
    # more prompts than a warp deals for itself, and contexts long enough that several CTAs share one
    seqs = [(4000 + 700 * (i % 5) if i % 60 == 7 else i % 37, (i * 7) % (nodes + 1)) for i in range(300)]
    b = Batch(seqs, mask="tree", seed=nodes, **kw)
    b.attend()
    b.check()
    w = torch.rand((len(seqs), b.hkv, b.max_len), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    before = w.clone()
    pcb.attention_weights(b.q, b.k, b.lse, w, decay=0.75, **b.args())
    pcb.ops_status(b.ws)
    check_weights(b, w, before, None, 0.75)


@pytest.mark.parametrize("hq", [4, 64])
def test_values_beyond_the_bounds_count_as_the_bounds(hq):
    b = Batch([(100, 4), (60, 2)], mask="tree", fill=0.0, hq=hq)
    spare = next(p for p in range(b.k.shape[0] // 16) if not (b.page_table == p).any())       # a page of zeros
    assert b.max_len == 104 and b.max_nodes == 4 and b.n_rows == 9
    got = []
    for ctx, first, pages in (([100, 0], [0, 4, 8], [spare, spare]), ([10 ** 9, -5], [-3, 4, 10 ** 6], [-7, 2 ** 31 - 1])):
        b.ctx_len.copy_(torch.tensor(ctx, dtype=torch.int32))
        b.row_start_d.copy_(torch.tensor(first, dtype=torch.int32))
        b.page_table[0, 2:4] = torch.tensor(pages, dtype=torch.int32)
        b.out.fill_(7.0)
        b.lse.fill_(7.0)
        b.attend()
        w = torch.full((2, b.hkv, b.max_len + 3), 7.0, device="cuda")
        pcb.attention_weights(b.q, b.k, b.lse, w, **b.args())
        pcb.ops_status(b.ws)
        assert (b.out[8:] == 7.0).all() and (b.lse[8:] == 7.0).all()           # the second prompt has four rows at most
        assert (w[0, :, 104:] == 7.0).all() and (w[1, :, 4:] == 7.0).all()
        got.append([x.clone() for x in (b.out, b.lse, w)])
    assert torch.isfinite(got[0][0].float()).all() and not torch.isnan(got[0][2]).any()
    assert all(torch.equal(x, y) for x, y in zip(*got))


def test_selection_and_moves_with_values_beyond_the_bounds():
    n, h, budget = 96, 2, 24
    gen = torch.Generator(device="cuda").manual_seed(2)
    w = torch.rand((3, h, n), generator=gen, device="cuda")
    pool = torch.randn((4 * n, h, 128), generator=gen, device="cuda").half()
    start = torch.tensor([0, n, 2 * n], dtype=torch.int32).cuda()
    got = []
    for length in ([n, 0, 40], [10 ** 9, -3, 40]):
        keep = torch.full((3, h, budget), 99, dtype=torch.int32, device="cuda")
        count = torch.full((3,), 99, dtype=torch.int32, device="cuda")
        pcb.select_slots(w, torch.tensor(length, dtype=torch.int32).cuda(), keep, count, sink=1, recent=5)
        got.append((keep, count))
    assert all(torch.equal(x, y) for x, y in zip(*got))
    assert got[0][1].tolist() == [budget, 0, budget]
    keep, count = got[0]
    moved = []
    for c in ([budget, 0, budget], [10 ** 9, -1, 2 ** 31 - 1]):
        k, v, ww = pool.clone(), -pool, w.clone()
        pcb.compact_slots(k, v, keep, torch.tensor(c, dtype=torch.int32).cuda(), max_len=n, weights=ww, ctx_start=start)
        moved.append((k, v, ww))
    assert all(torch.equal(x, y) for x, y in zip(*moved))
    for b in (0, 2):
        for g in range(h):
            at = keep[b, g].long()
            assert torch.equal(moved[0][0][b * n:b * n + budget, g], pool[b * n + at, g]) and torch.equal(moved[0][2][b, g, :budget], w[b, g, at])
            assert torch.equal(moved[0][0][b * n + budget:(b + 1) * n], pool[b * n + budget:(b + 1) * n])
    assert torch.equal(moved[0][0][n:2 * n], pool[n:2 * n]) and torch.equal(moved[0][0][3 * n:], pool[3 * n:])
