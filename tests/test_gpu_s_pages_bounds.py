"""Operators on pages: large offsets, values beyond the host's bounds, streams, graphs, shared workspaces, refusals of the binding."""
import numpy as np
import pytest

from oracle import pages as P
from paper_2601_11553_b200 import percache as pcb

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests.test_gpu_r_pages import F8, Batch, Forest, Rows, f64, i32, raw      # noqa: E402


def test_pages_past_32_bits():
    """Five gigabytes of pages, the last ones in use: written by an append, read by the attention, copied by a fork."""
    hkv, d, total = 8, 128, 155000
    pages = torch.zeros((1, total, hkv, 2, 16, d), dtype=torch.uint8, device="cuda").view(F8)
    scales = torch.zeros((1, total, hkv, 2), device="cuda")
    n = 300
    r = Rows([(0, n)], hq=16, hkv=hkv, cache="8bit")
    last = np.arange(total - 19, total).astype(np.int32)[::-1].copy()
    r.table, r.pages, r.scales = last[None], pages[0], scales[0]
    r.kw.update(pages=pages[0], scales=scales[0], page_table=torch.from_numpy(r.table).cuda())
    r.run()
    b = Batch([(n - 1, 1)], hq=16, hkv=hkv)
    b.pages, b.scales, b.table, b.page_table = pages[0], scales[0], r.table, r.kw["page_table"]
    b.attend()
    b.check()
    assert (f64(scales[0, last[:19].astype(np.int64)]) > 0).all()
    refs, free = torch.zeros(total, dtype=torch.int32, device="cuda"), torch.zeros(total, dtype=torch.int32, device="cuda")
    refs[torch.from_numpy(last.astype(np.int64)).cuda()] = 1
    free[0] = total - 25
    t = torch.zeros((2, 19), dtype=torch.int32, device="cuda")
    pcb.fork_pages(r.kw["page_table"], i32([19]), i32([n]), i32([0, 0]), t, i32([0, 0]), i32([0, 0]), refs, free, i32([1]), i32([0]),
                   pools=[pages, scales], workspace=b.ws)
    torch.cuda.synchronize()
    assert t[0].tolist() == last.tolist() and t[1].tolist() == last[:18].tolist() + [total - 25]
    assert torch.equal(pages[0, total - 25].view(torch.uint8), pages[0, int(last[18])].view(torch.uint8)) and torch.equal(scales[0, total - 25], scales[0, int(last[18])])
    assert refs[total - 25].item() == 1 and int(refs.sum()) == 18 * 2 + 1 + 1


@pytest.mark.parametrize("hq", [4, 64])
def test_attention_with_values_beyond_the_bounds(hq):
    b = Batch([(100, 4), (60, 2)], mask="tree", hq=hq)
    b.pages.view(torch.uint8)[torch.from_numpy(b.table[1, :4].astype(np.int64)).cuda(), :, :, :, :] = 0x20
    b.scales[:] = 0.01
    got = []
    for ctx, first in (([100, 0], [0, 4, 8]), ([10 ** 9, -5], [-3, 4, 10 ** 6])):
        b.ctx_len.copy_(i32(ctx))
        b.row_start_d.copy_(i32(first))
        b.out.fill_(7.0), b.lse.fill_(7.0)
        b.attend()
        assert (b.out[8:] == 7.0).all() and (b.lse[8:] == 7.0).all()           # the second prompt has four rows at most
        got.append([b.out.clone(), b.lse.clone()])
    assert torch.isfinite(got[0][0].float()).all() and all(torch.equal(x, y) for x, y in zip(*got))


@pytest.mark.parametrize("cache", ["8bit", "pages", "slots"])
@pytest.mark.parametrize("new, hq, hkv", [(3, 4, 2), (60, 4, 2), (1500, 47, 24)])          # the last: enough for the kernel of long prompts
def test_append_with_values_beyond_the_bounds(cache, new, hq, hkv):
    """Slots in use beyond max_len (the prompt's end), negative ones (none), rows past the last (all there are)."""
    got = []
    for ctx, first in (([40, 0], [0, new, 2 * new + 2]), ([10 ** 9, -5], [-3, new, 10 ** 6])):
        r = Rows([(40, new), (30, new)], cache=cache, pad_rows=2, hq=hq, hkv=hkv)
        r.kw["max_len"] = 40 + new
        r.kw["ctx_len"].copy_(i32(ctx)), r.kw["row_start"].copy_(i32(first))
        if cache != "slots":
            r.table[1] = r.table[1].clip(0, 5)                  # every page that its rows may reach is one of the pool's
            r.table[1, :] = np.arange(r.table.shape[1]) % len(r.before[0]) if cache == "8bit" else np.arange(r.table.shape[1])
            r.kw["page_table"].copy_(torch.from_numpy(r.table))
            r.kw["page_table"][0] = -1                          # and the first prompt's are not
        r.run()
        got.append([r.q_out.clone()] + [x.clone() for x in ([r.pages.view(torch.uint8), r.scales] if cache == "8bit" else r.pool)])
    assert all(torch.equal(x, y) for x, y in zip(*got))
    assert torch.isfinite(got[0][0].float()).all()


# Batches that the kernel of many rows takes: units that begin and end inside a prompt's pages, prompts shorter than a unit, heads that do not divide
# among the warps, rows ahead of and behind the prompts'.
MANY = [
    dict(seqs=[(5, 8300)], hq=16, hkv=8), dict(seqs=[(0, 3000), (117, 2500), (16, 2801)], hq=16, hkv=8, norm=False, rope=False),
    dict(seqs=[(i % 37, 64 + i % 51) for i in range(61)], hq=30, hkv=10, position=True), dict(seqs=[(0, 1), (3, 4000), (7, 0), (21, 5), (8, 300)], hq=45, hkv=9),
    dict(seqs=[(2, 5400)], hq=33, hkv=9, d=64, dtype="f16"), dict(seqs=[(31, 2200), (0, 3300)], hq=0, hkv=30, d=64, rope=False), dict(seqs=[(9, 90000)], hq=1, hkv=1, d=64),
]


@pytest.mark.parametrize("case", range(len(MANY)))
@pytest.mark.parametrize("cache, dtype", [("8bit", "bf16"), ("8bit", "f16"), ("pages", "bf16"), ("slots", "f16")])
def test_append_of_many_rows_matches_the_oracle(case, cache, dtype):
    kw = {"dtype": dtype, **MANY[case]}
    no_q = kw["hq"] == 0
    r = Rows(cache=cache, seed=case, **{**kw, "hq": kw["hq"] or 2})
    r.run(q=not no_q)
    r.check(q=not no_q)


@pytest.mark.parametrize("hkv, n, rows", [(2, 1000, 66), (6, 340, 67)])
def test_pages_in_turn_with_an_odd_number_of_heads_a_warp(hkv, n, rows):
    """The warps of a page's halves go from a page's last head to the next page's first: one and three heads each, values of very different sizes."""
    r = Rows([(3 + 5 * i % 16, rows) for i in range(n)], hkv=hkv, d=64, norm=False, rope=False, spread=4.0)
    r.run(q=False)
    r.check(q=False)


def test_many_rows_in_place_beside_other_prompts_rows():
    r = Rows([(3, 4000), (50, 4500)], hq=16, hkv=8, packed=False)
    q = r.q.clone()
    pcb.append_rows(q, r.k, r.v, q, **r.kw)
    r.q_out[:r.n] = q[:r.n]
    assert torch.equal(q[r.n:], r.q[r.n:])
    r.check()
    first = raw(r.pages).copy(), r.scales.clone()
    for _ in range(3):                                          # the same rows again, over pages whose scales are theirs already
        r.run()
        assert np.array_equal(raw(r.pages), first[0]) and torch.equal(r.scales, first[1])


def test_large_and_odd_values_among_many_rows():
    r = Rows([(3, 8300)], hq=16, hkv=8, norm=False, rope=False)
    r.k[0, 0, 3], r.k[900, 7, 127], r.k[901, 1, 64], r.v[8299, 5, 0], r.v[40, 2, 9] = float("inf"), float("nan"), float("-inf"), 3e38, float("nan")
    r.k[16 * 7 - 3:16 * 8 - 3] = 0.0
    r.run()
    r.check()
    r = Rows([(3, 8300)], hq=16, hkv=8, dtype="f16", cache="slots")
    r.k[500] = 60000.0
    r.kw["k_gain"] = torch.full_like(r.gains[1], 3e5)
    r.run()
    k = f64(r.pool[0])[int(r.start[0]) + 503]
    assert np.isfinite(k).all() and np.abs(k).max() == 65504


def test_twenty_thousand_prompts():
    r = Rows([(i % 16, 1) for i in range(20000)], hq=1, hkv=1, d=64, cache="8bit")
    r.run()
    for b, c, n, rr, wq, wk, wv in r.wanted():
        if b % 997 == 0:
            page, s = r.table[b, c // 16], f64(r.scales)[r.table[b, c // 16]]
            got = P.VALUES[raw(r.pages[int(page)])[0, :, c % 16]]
            assert (np.abs(got[0] * s[0, 0] - wk[0, 0]) <= np.maximum(np.abs(wk[0, 0]) * 2.0 ** -4, s[0, 0] * 2.0 ** -10) * 1.01 + 1e-3).all()
            assert (np.abs(got[1] * s[0, 1] - wv[0, 0]) <= np.maximum(np.abs(wv[0, 0]) * 2.0 ** -4, s[0, 1] * 2.0 ** -10)).all()
    eps = torch.finfo(r.q.dtype).eps / 2
    q = f64(r.q_out)[:r.n]
    r.near(q, np.concatenate([x[4] for x in r.wanted()]), eps, "q")


def test_calls_without_a_stream_take_the_current_one_and_two_workspaces_work_at_once():
    b, c = Batch([(3000, 2), (77, 1)], seed=1), Batch([(2000, 20)], mask="tree", seed=2, dtype="f16")
    f = Forest([70, 37], shared=2)
    r = Rows([(5, 40)])
    side = torch.cuda.Stream()
    q, k = torch.zeros_like(b.q), torch.zeros_like(r.k)
    t = dict(page_table=i32(f.table), held=i32(f.held), length=i32([0, 0]), parent=i32([1, 1, 0]), table_out=torch.zeros((3, f.width), dtype=torch.int32, device="cuda"),
             held_out=i32([0] * 3), length_out=i32([0] * 3), refs=i32(f.refs), free_list=i32(f.free + [0] * (f.total - len(f.free))), free_count=i32([len(f.free)]), missing=i32([9]))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        q.copy_(b.q), k.copy_(r.k), t["length"].copy_(i32(f.length))
        pcb.tree_attention_8bit(q, b.pages, b.scales, b.out, b.lse, ctx_len=b.ctx_len, row_start=b.row_start_d, page_table=b.page_table, max_nodes=b.max_nodes,
                                max_len=b.max_len, workspace=b.ws)
        pcb.append_rows(r.q, k, r.v, r.q_out, **r.kw)
        pcb.fork_pages(**t, pools=f.pools, room=1, workspace=f.ws)
    c.attend()
    torch.cuda.synchronize()
    b.check(), c.check(), r.check()
    want = P.fork(f.table, f.held, f.length, [1, 1, 0], f.width, f.refs, f.free, 1, f.total)
    assert t["held_out"].tolist() == want[1] and t["refs"].tolist() == want[3] and t["missing"].item() == want[5]
    assert t["length_out"].tolist() == want[2]


def test_one_workspace_for_all_calls_of_a_stream():
    """A fork leaves its plan in the workspace, the attention its parts: neither minds."""
    b = Batch([(5000, 3), (900, 2)], seed=3)
    f = Forest([70, 37, 200], shared=2)
    f.ws = b.ws
    for i in range(3):
        b.out.fill_(7.0), b.lse.fill_(7.0)
        b.attend()
        b.check()
        f.fork([0, 1, 1, 2], in_place=i % 2 == 1)
        f.table, f.held, f.length = f.table[:3], f.held[:3], f.length[:3]
        f.refs = [sum(p in row[:h] for row, h in zip(f.table, f.held)) for p in range(f.total)]
        f.free = [p for p in range(f.total) if f.refs[p] == 0]
    pcb.ops_status(b.ws)


def test_forks_are_captured_and_replayed():
    f = Forest([70, 37, 50], shared=2)
    n = f.total
    t = dict(page_table=i32(f.table), held=i32(f.held), length=i32(f.length), parent=i32([0, 0, 0, 0]), table_out=torch.zeros((4, f.width), dtype=torch.int32, device="cuda"),
             held_out=i32([0] * 4), length_out=i32([0] * 4), refs=i32(f.refs), free_list=i32(f.free + [-7] * (n - len(f.free))), free_count=i32([len(f.free)]), missing=i32([9]))
    outs = dict(refs_out=i32([0] * n), free_list_out=i32([0] * n), free_count_out=i32([0]))
    start = [p.clone() for p in f.pools]
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        pcb.fork_pages(**t, **outs, pools=f.pools, room=1, workspace=f.ws)
    for parent in ([2, 1, 2, 0], [1, 1, 1, 7]):
        t["parent"].copy_(i32(parent))
        for p, x in zip(f.pools, start):
            p.copy_(x)
        g.replay()
        torch.cuda.synchronize()
        table, held, length, refs, free, missing, copies = P.fork(f.table, f.held, f.length, parent, f.width, f.refs, f.free, 1, n)
        assert t["table_out"].tolist() == [x + [-1] * (f.width - len(x)) for x in table] and t["held_out"].tolist() == held
        assert outs["refs_out"].tolist() == refs and outs["free_list_out"].tolist()[:len(free)] == free and outs["free_count_out"].tolist() == [len(free)]
        for p, x in zip(f.pools, start):
            want = x.clone()
            for a, b in copies:
                want[:, b] = x[:, a]
            assert torch.equal(p, want)


def test_gains_may_be_parameters():
    r = Rows([(3, 5)])
    r.kw["q_gain"], r.kw["k_gain"] = (torch.nn.Parameter(g.clone()) for g in r.gains)
    r.run()
    r.check()


def test_the_binding_refuses_tensors_that_do_not_fit():
    r = Rows([(3, 5)])

    def bad(match, **kw):
        args = {**dict(q=r.q, k=r.k, v=r.v, q_out=r.q_out), **r.kw, **kw}
        q, k, v, o = (args.pop(x) for x in ("q", "k", "v", "q_out"))
        with pytest.raises(ValueError, match=match):
            pcb.append_rows(q, k, v, o, **args)

    bad("q_out", q_out=None)
    bad("q_out", q=None)
    bad("v", v=r.v[:-1])
    bad("v", v=r.v.half())
    bad("k", k=r.k.float())
    bad("q", q=r.q[:-1])
    bad("q_out", q_out=r.q_out[:, :-1])
    bad("k", k=r.k.transpose(0, 1))
    bad("ctx_len", ctx_len=r.kw["ctx_len"].long())
    bad("row_start", row_start=r.kw["ctx_len"])
    bad("q_gain", q_gain=r.gains[0].half())
    bad("k_gain", k_gain=r.gains[0][:-1])
    bad("rope", rope=r.rope[:, :-1])
    bad("rope", rope=r.rope.transpose(0, 1))
    bad("position", position=r.kw["ctx_len"])
    bad("pools", pages=None)
    bad("pools", scales=None)
    bad("pools", k_pool=r.k, v_pool=r.v)
    bad("ctx_start", ctx_start=r.kw["ctx_len"])
    bad("pages", pages=r.pages[:, :, :, :8])
    bad("pages", pages=r.pages.transpose(1, 2))
    bad("pages", pages=r.pages.view(torch.uint8).view(torch.int8))
    bad("pages", pages=r.pages[:, :1], scales=r.scales[:, :1].contiguous())          # another number of heads
    bad("scales", scales=r.scales[:-1])
    bad("scales", scales=r.scales.double())
    bad("page_table", page_table=r.kw["page_table"].long())
    with pytest.raises(pcb.PerCacheError):                                              # strides that a page's copy cannot have
        big = torch.zeros((len(r.pages), 2 * 32 * 128 + 16), dtype=torch.uint8, device="cuda")
        pcb.append_rows(r.q, r.k, r.v, r.q_out, **{**r.kw, "pages": big.as_strided(r.pages.shape, (2 * 32 * 128 + 16,) + r.pages.stride()[1:])})
    b = Batch([(30, 2)])
    kw = dict(ctx_len=b.ctx_len, row_start=b.row_start_d, page_table=b.page_table, max_nodes=2, max_len=32, workspace=b.ws)
    for name, args in (("q", (b.q[:, :, :64], b.pages, b.scales, b.out, b.lse)), ("out", (b.q, b.pages, b.scales, b.out[:-1], b.lse)), ("lse", (b.q, b.pages, b.scales, b.out, b.lse[:-1])),
                       ("out", (b.q, b.pages, b.scales, b.out.half(), b.lse)), ("pages", (b.q, b.pages.float(), b.scales, b.out, b.lse))):
        with pytest.raises(ValueError, match=name):
            pcb.tree_attention_8bit(*args, **kw)
    with pytest.raises(pcb.PerCacheError):
        pcb.tree_attention_8bit(b.q, b.pages, b.scales, b.out, b.lse, **{**kw, "max_len": 33})
    f = Forest([20])
    n = f.total
    t = dict(page_table=i32(f.table), held=i32(f.held), length=i32(f.length), parent=i32([0]), table_out=torch.zeros((1, f.width), dtype=torch.int32, device="cuda"),
             held_out=i32([0]), length_out=i32([0]), refs=i32(f.refs), free_list=i32([0] * n), free_count=i32([0]), missing=i32([9]), pools=f.pools, workspace=f.ws)
    for name, x in (("length", i32([1, 2])), ("table_out", torch.zeros((2, 3), dtype=torch.int32, device="cuda")), ("held_out", i32([1, 2])),
                    ("free_list", i32([0] * (n + 1))), ("free_count", i32([1, 2])), ("missing", i32([])), ("pools", [f.pools[0][:, :-1]]), ("pools", [f.pools[0].transpose(0, 1)]),
                    ("pools", [f.pools[0].cpu()]), ("pools", [f.pools[0][..., ::2]]), ("pools", [f.pools[0]] * 9), ("workspace", f.ws.float())):
        with pytest.raises(ValueError, match=name):
            pcb.fork_pages(**{**t, name: x})
    with pytest.raises(ValueError, match="page_table"):
        pcb.fork_pages(**{**t, "held": i32([1, 2])})
    for name in ("refs", "free_list", "free_count"):                                    # each its own array, or none
        with pytest.raises(pcb.PerCacheError):
            pcb.fork_pages(**t, **{name + "_out": t[name].clone()})
    with pytest.raises(pcb.PerCacheError):
        pcb.fork_pages(**{**t, "table_out": t["page_table"]})


def test_heavier_pages_do_not_hide_lighter_ones():
    """Values of one page 2^40 times those of the others, at equal scores: weights and sums keep to what they stand for."""
    b = Batch([(200, 1)], q_scale=0.01)
    for p, e in ((3, 30.0), (5, -30.0)):
        b.scales[int(b.table[0, p]), :, 1] = 2.0 ** e
    b.attend()
    b.check()
