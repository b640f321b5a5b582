"""Operators on a decoding batch's cache against the float64 oracle.

Tolerances.  A score x = scale * sum q k over D products: fp32 accumulation is off by at most D * 2^-23 * scale * sum |q k|
(delta below; twice the bound of round-to-nearest, since a matrix unit may truncate), the exponential of a difference by another
2^-20 relative.  The softmax weights are rounded to the pools' type before they multiply V (half a step: eps / 2, relative), the output
is rounded once more, so an output element is off by at most (eps/2 + delta + 2^-19) * A + eps/2 * |out|, with A the
weighted average of |v|; the row sum is not rounded and the two error kinds of numerator and denominator double delta.  fp16 weights
below 2^-14 (relative to the largest, which the running reference keeps at or above 2^-8 of full scale) round to multiples of
2^-24: another 2^-16 * max |v| at the very most.
"""
import numpy as np
import pytest

from oracle import cache_ops as ops
from paper_2601_11553_b200 import percache as pcb

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def f64(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


class Batch:
    """A ragged batch over shared pools; seqs: [(ctx_len, nodes)].  mask: None (chain), "tree", "random" or "empty"."""

    def __init__(self, seqs, dtype="bf16", hq=4, hkv=2, d=128, paged=True, mask=None, seed=0, q_scale=1.0, pad_rows=3, wide=0,
                 fill=float("nan")):
        self.seqs, self.hq, self.hkv, self.d, self.paged = seqs, hq, hkv, d, paged
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        t = TYPES[dtype]
        lens = [c + n for c, n in seqs]
        self.max_len = max(max(lens, default=1), 1)
        self.max_nodes = max(max((n for _, n in seqs), default=1), 1)
        n_seqs = len(seqs)
        self.page_table = self.ctx_start = None
        if paged:
            pages = [-(-x // 16) for x in lens]
            total = sum(pages) + 2
            order = rng.permutation(total)
            table = np.full((n_seqs, -(-self.max_len // 16)), 10 ** 6, dtype=np.int32)     # entries that are never used point nowhere
            at = 0
            for b, p in enumerate(pages):
                table[b, :p] = order[at:at + p]
                at += p
            self.page_table = torch.from_numpy(table).cuda()
            self.rows = [(table[b, :pages[b], None].astype(np.int64) * 16 + np.arange(16)).reshape(-1)[:lens[b]] for b in range(n_seqs)]
            slots = total * 16
        else:
            start, at = [], 7
            for x in lens:
                start.append(at)
                at += x + 1
            self.ctx_start = torch.tensor(start, dtype=torch.int32).cuda()
            self.rows = [np.arange(start[b], start[b] + lens[b], dtype=np.int64) for b in range(n_seqs)]
            slots = at + 5
        # pools: rows no prompt owns hold `fill`; `wide` more elements between rows than the heads need
        def pool():
            x = torch.full((slots, hkv * d + wide), fill, dtype=t, device="cuda")
            own = np.concatenate(self.rows) if n_seqs else np.zeros(0, dtype=np.int64)
            if len(own):
                x[torch.from_numpy(own).cuda(), :hkv * d] = torch.randn((len(own), hkv * d), generator=gen, device="cuda").to(t)
            return x.as_strided((slots, hkv, d), (hkv * d + wide, d, 1))
        self.k, self.v = pool(), pool()
        self.row_start = np.concatenate([[0], np.cumsum([n for _, n in seqs])]).astype(np.int32)
        self.n = int(self.row_start[-1])
        self.n_rows = self.n + pad_rows
        big = (q_scale * torch.randn((self.n_rows, hq * d + wide), generator=gen, device="cuda")).to(t)
        self.q = big.as_strided((self.n_rows, hq, d), (hq * d + wide, d, 1))
        self.out = torch.full((self.n_rows, hq * d + wide), 7.0, dtype=t, device="cuda").as_strided((self.n_rows, hq, d), (hq * d + wide, d, 1))
        self.lse = torch.full((self.n_rows, hq), 7.0, device="cuda")
        self.node_mask = [None] * n_seqs
        self.mask = None
        if mask is not None:
            words = -(-self.max_nodes // 64)
            bits = np.zeros((self.n_rows, words), dtype=np.uint64)
            for b, (c, n) in enumerate(seqs):
                m = np.zeros((n, n), dtype=bool)
                for i in range(n):
                    if mask == "tree":
                        p = int(rng.integers(-1, i)) if i else -1
                        if p >= 0:
                            m[i] = m[p]
                        m[i, i] = True
                    elif mask == "random":
                        m[i] = rng.random(n) < 0.4
                self.node_mask[b] = m
                for i in range(n):
                    for j in np.flatnonzero(m[i]):
                        bits[self.row_start[b] + i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
                    # bits past the prompt's nodes mean nothing
                    for j in range(n, 64 * words):
                        bits[self.row_start[b] + i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
            self.mask = torch.from_numpy(bits.view(np.int64)).cuda()
        self.ctx_len = torch.tensor([c for c, _ in seqs], dtype=torch.int32).cuda()
        self.row_start_d = torch.from_numpy(self.row_start).cuda()
        self.ws = torch.zeros(pcb.OPS_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
        self.scale = d ** -0.5

    def args(self):
        return dict(ctx_len=self.ctx_len, row_start=self.row_start_d, mask=self.mask, page_table=self.page_table,
                    ctx_start=self.ctx_start, max_nodes=self.max_nodes, max_len=self.max_len, scale=self.scale, workspace=self.ws)

    def attend(self, **kw):
        pcb.tree_attention(self.q, self.k, self.v, self.out, self.lse, **{**self.args(), **kw})
        pcb.ops_status(self.ws)

    def part(self, b):
        r0, r1 = int(self.row_start[b]), int(self.row_start[b + 1])
        at = torch.from_numpy(self.rows[b]).cuda()
        return r0, r1, f64(self.k[at]), f64(self.v[at])

    def check(self, pad_untouched=True):
        q, out, lse = f64(self.q), f64(self.out), f64(self.lse)
        eps = torch.finfo(self.q.dtype).eps / 2
        for b, (c, n) in enumerate(self.seqs):
            if n == 0:
                continue
            r0, r1, k, v = self.part(b)
            want, wlse, mean_abs = ops.tree_attention(q[r0:r1], k, v, c, self.node_mask[b], self.scale)
            seen = ops.sees(n, c, self.node_mask[b])
            delta = self.delta(q[r0:r1], k, seen)[:, :, None]
            vmax = max((np.abs(x[np.isfinite(x)]).max(initial=0.0) for x in v), default=0.0)
            tol = (eps + 2 * delta + 2.0 ** -18) * mean_abs + eps * np.abs(want) + 2.0 ** -16 * vmax * (self.q.dtype == torch.float16) + 1e-30
            fine = np.isfinite(want)
            assert np.array_equal(np.isnan(out[r0:r1]), np.isnan(want)), b
            assert np.array_equal(out[r0:r1][~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), b
            bad = np.abs(out[r0:r1] - want)[fine] > tol[fine]
            assert not bad.any(), (b, c, n, np.abs(out[r0:r1] - want)[fine].max(), int(bad.sum()), bad.size)
            assert np.array_equal(np.isnan(lse[r0:r1]), np.isnan(wlse))
            lf = np.isfinite(wlse)
            assert np.array_equal(lse[r0:r1][~lf & ~np.isnan(wlse)], wlse[~lf & ~np.isnan(wlse)])
            ltol = delta[:, :, 0] + 2.0 ** -20 * (np.abs(np.where(lf, wlse, 0)) + 4)
            assert (np.abs(lse[r0:r1] - wlse)[lf] <= ltol[lf]).all(), (b, np.abs(lse[r0:r1] - wlse)[lf].max())
        if pad_untouched:
            assert (out[self.n:] == 7.0).all() and (lse[self.n:] == 7.0).all()

    def delta(self, q, k, seen):
        """Bound on a score's absolute error, per (node, head): over the slots it sees."""
        group = self.hq // self.hkv
        with np.errstate(invalid="ignore", over="ignore"):
            x = np.einsum("nhd,thd->nht", np.abs(q), np.repeat(np.abs(k), group, axis=1)) * self.scale
        x = np.where(np.isfinite(x) & seen[:, None, :], x, 0)
        return x.max(axis=2, initial=0.0) * self.d * 2.0 ** -23


SHAPES = [
    # one token: the decode step, at lengths around the block and page borders
    dict(seqs=[(0, 1)]), dict(seqs=[(1, 1)]), dict(seqs=[(15, 1)]), dict(seqs=[(16, 1)], dtype="f16"), dict(seqs=[(126, 1)]),
    dict(seqs=[(127, 1)], dtype="f16"), dict(seqs=[(128, 1)]), dict(seqs=[(129, 1)], paged=False), dict(seqs=[(255, 1)]),
    dict(seqs=[(256, 1)], paged=False, dtype="f16"), dict(seqs=[(1000, 1)], hq=16, hkv=8),
    # head layouts: one to 128 query heads a KV head, both head sizes
    dict(seqs=[(200, 3)], hq=1, hkv=1), dict(seqs=[(200, 3)], hq=3, hkv=1, mask="tree"), dict(seqs=[(200, 5)], hq=14, hkv=2, dtype="f16"),
    dict(seqs=[(77, 9)], hq=128, hkv=1, mask="tree"), dict(seqs=[(300, 2)], hq=100, hkv=2, d=64), dict(seqs=[(300, 40)], hq=8, hkv=8, d=64, dtype="f16", mask="tree"),
    dict(seqs=[(513, 33)], hq=5, hkv=5, d=64, paged=False, mask="random"),
    # trees: around the word and tile borders, up to the most nodes
    dict(seqs=[(100, 63)], mask="tree"), dict(seqs=[(100, 64)], mask="tree", dtype="f16"), dict(seqs=[(100, 65)], mask="tree"),
    dict(seqs=[(90, 128)], mask="tree", hq=4, hkv=4), dict(seqs=[(333, 256)], mask="tree", dtype="f16"), dict(seqs=[(0, 256)], mask="tree"),
    dict(seqs=[(5, 200)], mask="random", paged=False), dict(seqs=[(640, 130)], hq=6, hkv=2), dict(seqs=[(0, 17)]),
    dict(seqs=[(0, 40)], mask="empty"), dict(seqs=[(3, 40)], mask="empty"), dict(seqs=[(0, 70)], mask="random", dtype="f16"),
    # ragged batches, prompts without nodes and without context among them
    dict(seqs=[(700, 1), (3, 12), (0, 1), (129, 30), (64, 0), (2000, 7)], mask="tree"),
    dict(seqs=[(700, 1), (3, 12), (0, 0), (129, 30), (64, 0), (2000, 7)], mask="tree", paged=False, dtype="f16", hq=8),
    dict(seqs=[(i % 37, 1 + i % 3) for i in range(300)], hq=2, hkv=1, mask="tree"),
    dict(seqs=[(1500 + 131 * i, 1) for i in range(9)], hq=16, hkv=8, paged=False, dtype="f16"),
    # long contexts: split over many blocks
    dict(seqs=[(20000, 1)], hq=2, hkv=1), dict(seqs=[(33024, 4)], hq=4, hkv=1, dtype="f16", paged=False), dict(seqs=[(9000, 48)], mask="tree"),
    # rows further apart than their heads need
    dict(seqs=[(300, 6), (40, 2)], wide=8, mask="tree"), dict(seqs=[(300, 6), (40, 2)], wide=136, paged=False, dtype="f16", d=64),
    # large scores: the softmax is nearly one slot
    dict(seqs=[(400, 20)], q_scale=12.0, mask="tree"), dict(seqs=[(1200, 3)], q_scale=30.0, dtype="f16"),
]


@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_tree_attention_matches_the_oracle(case):
    b = Batch(seed=case, **SHAPES[case])
    b.attend()
    b.check()


def test_tree_attention_is_the_same_every_time():
    b = Batch([(5000, 9), (130, 2), (0, 1)], mask="tree", hq=8)
    b.attend()
    first, lse = b.out.clone(), b.lse.clone()
    for _ in range(5):
        b.out.fill_(7.0)
        b.attend()
        assert torch.equal(first, b.out) and torch.equal(lse, b.lse)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_row_does_not_see_may_hold_anything(dtype, bad):
    # node 4 is seen by itself alone; the pools' other rows hold the same bad value already (fill)
    b = Batch([(250, 6), (17, 1)], dtype=dtype, mask="tree", fill=bad)
    for i in range(6):
        for j in range(6):
            b.node_mask[0][i, j] = i == j or (j == 0 and i != 4)
    words = [sum(1 << j for j in range(6) if b.node_mask[0][i, j]) for i in range(6)]
    b.mask[:6, 0] = torch.tensor(words, dtype=torch.int64).cuda()
    row = int(b.rows[0][254])
    b.v[row, 0, 3] = bad
    b.v[row, 1, :] = bad
    b.attend()
    b.check()                                   # node 4 shows the bad value where V has it, nobody else does
    assert not torch.isfinite(b.out[4, 0, 3]) and torch.isfinite(b.out[[0, 1, 2, 3, 5]].float()).all()
    b.k[row] = bad
    b.attend()
    assert torch.isfinite(b.out[[0, 1, 2, 3, 5]].float()).all()


def test_a_bad_value_in_the_context_reaches_every_row_of_its_heads():
    b = Batch([(300, 4)], mask="tree")
    b.v[int(b.rows[0][10]), 1, 5] = float("nan")
    b.attend()
    b.check()
    assert torch.isnan(b.out[:4, 2:, 5]).all() and torch.isfinite(b.out[:4, :2].float()).all()


def test_tree_attention_without_lse_and_on_another_stream():
    b = Batch([(900, 5), (40, 1)], mask="tree")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pcb.tree_attention(b.q, b.k, b.v, b.out, None, **b.args(), stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    lse = b.lse.clone()
    assert (lse == 7.0).all()
    first = b.out.clone()
    b.attend()
    b.check()
    assert torch.equal(first, b.out)


def test_a_captured_call_follows_lengths_tables_and_masks():
    b = Batch([(700, 6), (90, 6)], mask="tree")
    w = torch.zeros((2, b.hkv, b.max_len), device="cuda")
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b.attend(stream=side.cuda_stream)                   # first launches outside the capture
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            pcb.tree_attention(b.q, b.k, b.v, b.out, b.lse, **b.args(), stream=side.cuda_stream)
            pcb.attention_weights(b.q, b.k, b.lse, w, **b.args(), stream=side.cuda_stream)
    torch.cuda.synchronize()
    for seqs in ([(600, 3), (11, 5)], [(0, 1), (690, 6)], [(706, 0), (94, 2)]):
        c = Batch(seqs, mask="tree", seed=5, pad_rows=12 - sum(n for _, n in seqs))
        c.max_len, c.max_nodes = b.max_len, b.max_nodes
        # the new batch's data in the captured call's arrays
        table = torch.zeros_like(b.page_table)
        table[:, :c.page_table.shape[1]] = c.page_table
        b.page_table.copy_(torch.where(table >= b.k.shape[0] // 16, torch.zeros_like(table), table))
        assert c.k.shape[0] <= b.k.shape[0]
        b.k[:c.k.shape[0]] = c.k
        b.v[:c.v.shape[0]] = c.v
        b.q[:12] = c.q[:12]
        b.mask.zero_()
        b.mask[:12] = c.mask[:12]
        b.ctx_len.copy_(c.ctx_len)
        b.row_start_d.copy_(c.row_start_d)
        b.out.fill_(7.0)
        b.lse.fill_(7.0)
        w.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        b.seqs, b.rows, b.row_start, b.node_mask, b.n = c.seqs, c.rows, c.row_start, c.node_mask, c.n
        b.check()
        check_weights(b, w, torch.zeros_like(w), None, 1.0)


def test_offsets_past_32_bits():
    # 4096 rows of 1.3 M elements: the pool's last rows lie past 2^32 elements
    stride, slots = 1310720, 4096
    flat = torch.zeros(stride * (slots - 1) + 256, dtype=torch.bfloat16, device="cuda")
    k = flat.as_strided((slots, 2, 128), (stride, 128, 1))
    b = Batch([(300, 4)], mask="tree")
    order = np.random.default_rng(3).permutation(slots // 16)[:19]
    order[-1] = slots // 16 - 1
    rows = (order[:, None] * 16 + np.arange(16)).reshape(-1)[:304]
    at = torch.from_numpy(b.rows[0]).cuda()
    to = torch.from_numpy(rows).cuda()
    k[to] = b.k[at]
    table = torch.zeros_like(b.page_table)
    table[0, :19] = torch.from_numpy(order.astype(np.int32)).cuda()
    b.attend()
    want = b.out.clone()
    b.k, b.v, b.page_table, b.rows = k, k, table, [rows]
    b.out.fill_(7.0)
    b.attend()
    b.check()
    assert not torch.equal(want, b.out)
    w = torch.zeros((1, 2, b.max_len), device="cuda")
    pcb.attention_weights(b.q, b.k, b.lse, w, **b.args())
    check_weights(b, w, torch.zeros_like(w), None, 1.0)


def test_lengths_and_pages_outside_their_bounds_are_clamped_and_harmless():
    b = Batch([(100, 4), (60, 2)], mask="tree", fill=0.0)
    b.ctx_len.copy_(torch.tensor([10 ** 9, -5], dtype=torch.int32))
    b.page_table[0, 2] = -7
    b.page_table[0, 3] = 2 ** 31 - 1
    b.row_start_d.copy_(torch.tensor([-3, 4, 10 ** 6], dtype=torch.int32))
    b.attend()
    w = torch.zeros((2, b.hkv, b.max_len), device="cuda")
    pcb.attention_weights(b.q, b.k, b.lse, w, **b.args())
    torch.cuda.synchronize()


@pytest.mark.parametrize("page", [-1, -2 ** 31 + 1, -2 ** 31, 2 ** 30 + 1, 2 ** 31 - 1])
@pytest.mark.parametrize("n", [2, 40])
def test_a_page_outside_the_pool_reads_as_zeros(page, n):
    b = Batch([(200, n), (60, 2)], mask="tree", fill=0.0)
    spare = next(p for p in range(b.k.shape[0] // 16) if not (b.page_table == p).any())       # a page of zeros
    got = []
    for p in (spare, page):
        b.page_table[0, 3] = p
        b.attend()
        w = torch.zeros((2, b.hkv, b.max_len), device="cuda")
        pcb.attention_weights(b.q, b.k, b.lse, w, **b.args())
        got.append([x.clone() for x in (b.out, b.lse, w)])
    assert all(torch.equal(x, y) for x, y in zip(*got))


def check_weights(b, got, before, use, decay):
    q, lse, got, before = f64(b.q), b.lse.cpu().numpy(), f64(got), f64(before)
    for s, (c, n) in enumerate(b.seqs):
        r0, r1, k, _ = b.part(s)
        t = c + n
        u = None if use is None else use[r0:r1]
        want = ops.attention_weights(q[r0:r1], k, lse[r0:r1], u, c, b.node_mask[s], b.scale, before[s, :, :t], decay)
        seen = ops.sees(n, c, b.node_mask[s])
        delta = float(b.delta(q[r0:r1], k, seen).max(initial=0.0))
        big = float(np.abs(lse[r0:r1][np.isfinite(lse[r0:r1])]).max(initial=0.0)) + delta * 2 ** 23 / b.d
        # every term is off by its exponent's error (the score's, and rounding the difference at the size of its operands);
        # the sum of up to n * group + 1 terms by their number of roundings
        tol = want * (2 * delta + 2.0 ** -21 * (big + 4) + (n * b.hq // b.hkv + 2) * 2.0 ** -23) + 1e-30
        assert np.array_equal(np.isnan(got[s, :, :t]), np.isnan(want))
        ok = ~np.isnan(want)
        assert (np.abs(got[s, :, :t] - want)[ok] <= tol[ok]).all(), (s, np.abs(got[s, :, :t] - want)[ok].max())
        assert np.array_equal(got[s, :, t:], before[s, :, t:])


@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_attention_weights_match_the_oracle(case):
    b = Batch(seed=100 + case, **SHAPES[case])
    b.attend()
    gen = torch.Generator(device="cuda").manual_seed(case)
    w = torch.rand((len(b.seqs), b.hkv, b.max_len + case % 3), generator=gen, device="cuda")
    before = w.clone()
    use = None
    if case % 3:
        use = (torch.rand(b.n_rows, generator=gen, device="cuda") < 0.5).to(torch.uint8)
    decay = (1.0, 0.75, 0.0)[case % 3]
    pcb.attention_weights(b.q, b.k, b.lse, w, use=use, decay=decay, **b.args())
    pcb.ops_status(b.ws)
    check_weights(b, w, before, None if use is None else use.cpu().numpy(), decay)
    if case % 5 == 0:                                   # another array, and the same again
        out = before.clone()
        pcb.attention_weights(b.q, b.k, b.lse, before, out, use=use, decay=decay, **b.args())
        assert torch.equal(out, w)


def test_rows_that_do_not_count_may_hold_anything():
    b = Batch([(200, 6), (17, 3)], mask="tree", hq=8)
    b.attend()
    use = torch.tensor([1, 0, 1, 1, 0, 1, 0, 1, 1, 1, 1, 1], dtype=torch.uint8).cuda()
    b.q[1] = float("nan")
    b.q[4] = float("inf")
    b.q[6] = float("nan")
    b.lse[1] = float("nan")
    b.lse[4] = -float("inf")
    w = torch.zeros((2, b.hkv, b.max_len), device="cuda")
    pcb.attention_weights(b.q, b.k, b.lse, w, use=use, **b.args())
    assert torch.isfinite(w).all()
    check_weights(b, w, torch.zeros_like(w), use.cpu().numpy(), 1.0)


@pytest.mark.parametrize("n,budget,sink,recent", [(1, 1, 0, 0), (5, 8, 2, 2), (8, 8, 0, 0), (9, 8, 0, 0), (100, 1, 0, 0), (100, 1, 1, 0),
                                                  (100, 50, 25, 25), (1024, 100, 4, 16), (1025, 1024, 0, 1), (2112, 1024, 4, 128),
                                                  (5000, 33, 0, 0), (33024, 8192, 16, 1000), (40000, 39999, 1, 1)])
@pytest.mark.parametrize("kind", ["random", "ties", "odd"])
def test_select_slots_matches_the_oracle(n, budget, sink, recent, kind):
    rng = np.random.default_rng(n + budget)
    lens = [n, max(0, n - 3), 0, n // 2]
    h = 3
    w = rng.random((len(lens), h, n + 5)).astype(np.float32) ** 4
    if kind == "ties":
        w = np.round(w * 4).astype(np.float32)
    if kind == "odd":
        at = rng.random(w.shape)
        w[at < 0.1] = np.nan
        w[(at >= 0.1) & (at < 0.15)] = np.inf
        w[(at >= 0.15) & (at < 0.2)] = -np.inf
        w[(at >= 0.2) & (at < 0.4)] = -0.0
        w[(at >= 0.4) & (at < 0.6)] = 0.0
        w[(at >= 0.6) & (at < 0.7)] *= -1
    keep = torch.full((len(lens), h, budget), 99, dtype=torch.int32, device="cuda")
    count = torch.full((len(lens),), 99, dtype=torch.int32, device="cuda")
    pcb.select_slots(torch.from_numpy(w).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), keep, count, sink=sink, recent=recent, max_len=n)
    keep, count = keep.cpu().numpy(), count.cpu().numpy()
    for b, m in enumerate(lens):
        assert count[b] == min(m, budget)
        for g in range(h):
            want = ops.select_slots(w[b, g], m, budget, sink, recent)
            assert keep[b, g, :len(want)].tolist() == want
            assert (keep[b, g, len(want):] == -1).all()


def _pools(slots, hkv, d, dtype, wide=0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randint(-30000, 30000, (slots, hkv * d + wide), generator=gen, device="cuda", dtype=torch.int16).view(TYPES[dtype])
            .as_strided((slots, hkv, d), (hkv * d + wide, d, 1)) for _ in range(2)]


@pytest.mark.parametrize("paged", [True, False])
@pytest.mark.parametrize("lens,budget,hkv,d,dtype,wide,shared,with_first", [
    ([1], 1, 1, 128, "f16", 0, False, False), ([200, 33, 0, 77], 40, 2, 128, "bf16", 0, False, False),
    ([2112], 1024, 8, 128, "bf16", 0, False, False), ([5000, 100], 4999, 3, 64, "f16", 8, False, False),
    ([700, 650], 40, 2, 128, "bf16", 136, True, True), ([33024], 8192, 2, 128, "f16", 0, False, False)])
def test_compact_slots_in_place_and_to_another_place(paged, lens, budget, hkv, d, dtype, wide, shared, with_first):
    rng = np.random.default_rng(sum(lens) + budget)
    n, max_len = len(lens), max(lens)
    k, v = _pools((sum(-(-x // 16) for x in lens) * 2 + 3) * 16, hkv, d, dtype, wide)
    first = [x - 50 if with_first else 0 for x in lens]
    heads = 1 if shared else hkv
    keep = np.full((n, heads, budget), -1, dtype=np.int32)
    count = np.array([min(budget, x - f) for x, f in zip(lens, first)], dtype=np.int32)
    for b, x in enumerate(lens):
        for g in range(heads):
            keep[b, g, :count[b]] = np.sort(rng.permutation(np.arange(first[b], x))[:count[b]])
    w = torch.rand((n, hkv, max_len), device="cuda")
    if paged:
        width = -(-max_len // 16)
        order = rng.permutation(k.shape[0] // 16)
        src, dst, at = np.zeros((n, width), dtype=np.int32), np.zeros((n, width), dtype=np.int32), 0
        for t in (src, dst):
            for b, x in enumerate(lens):
                t[b, :-(-x // 16)] = order[at:at - (-x // 16)]
                at += -(-x // 16)
        place = lambda t, b, s: t[b, s // 16].astype(np.int64) * 16 + s % 16             # noqa: E731
        src_kw, dst_kw = dict(page_table=torch.from_numpy(src).cuda()), dict(dst_page_table=torch.from_numpy(dst).cuda())
    else:
        src = np.concatenate([[2], 2 + np.cumsum(lens)]).astype(np.int32)[:n]
        dst = (src + sum(lens)).astype(np.int32)
        place = lambda t, b, s: t[b].astype(np.int64) + s                                # noqa: E731
        src_kw, dst_kw = dict(ctx_start=torch.from_numpy(src).cuda()), dict(dst_start=torch.from_numpy(dst).cuda())
    fd = torch.tensor(first, dtype=torch.int32).cuda() if with_first else None
    for to, kw in ((dst, {**src_kw, **dst_kw}), (src, src_kw)):
        wants = []
        for x in (k, v):
            bits = x.contiguous().view(torch.int16).cpu().numpy()
            want = bits.copy()
            for b in range(n):
                for g in range(hkv):
                    s = keep[b, 0 if shared else g, :count[b]].astype(np.int64)
                    if len(s):
                        want[place(to, b, first[b] + np.arange(len(s))), g] = bits[place(src, b, s), g]
            wants.append(want)
        ww = w.cpu().numpy().copy()
        for b in range(n):
            for g in range(hkv):
                s = keep[b, 0 if shared else g, :count[b]]
                ww[b, g, first[b]:first[b] + len(s)] = w.cpu().numpy()[b, g, s]
        w_out = w.clone()
        pcb.compact_slots(k, v, torch.from_numpy(keep).cuda(), torch.from_numpy(count).cuda(), max_len=max_len, weights=w_out, first=fd, **kw)
        for x, want in zip((k, v), wants):
            assert np.array_equal(x.contiguous().view(torch.int16).cpu().numpy(), want)
        assert np.array_equal(w_out.cpu().numpy(), ww)


def test_compact_leaves_out_what_is_out_of_range():
    k, v = _pools(64, 2, 128, "bf16")
    k0, v0 = k.clone(), v.clone()
    keep = torch.tensor([[[-1, 1 << 20, 64, 5], [-7, 99, 1000, 2 ** 31 - 1]]], dtype=torch.int32).cuda()
    count = torch.tensor([1000], dtype=torch.int32).cuda()
    table = torch.tensor([[0, 10 ** 6, -1, 3]], dtype=torch.int32).cuda()
    pcb.compact_slots(k, v, keep, count, max_len=64, page_table=table)
    k0[3, 0] = k0[5, 0]
    v0[3, 0] = v0[5, 0]
    assert torch.equal(k.view(torch.int16), k0.view(torch.int16)) and torch.equal(v.view(torch.int16), v0.view(torch.int16))


def test_pools_smaller_than_a_block_and_a_single_row():
    b = Batch([(3, 1)], paged=False, hq=4, hkv=2, pad_rows=0)
    assert b.k.shape[0] < 128
    odd = torch.empty(2051, dtype=torch.bfloat16, device="cuda").as_strided((1, 4, 128), (2051, 128, 1))     # one row: its stride means nothing
    odd.copy_(b.q)
    b.q = odd
    b.attend()
    b.check()
    w = torch.zeros((1, 2, b.max_len), device="cuda")
    pcb.attention_weights(b.q, b.k, b.lse, w, **b.args())
    check_weights(b, w, torch.zeros_like(w), None, 1.0)


def test_the_binding_refuses_tensors_that_do_not_fit():
    b = Batch([(300, 3), (5, 1)], mask="tree")
    good = dict(b.args())

    def refused(match, q=b.q, k=b.k, v=b.v, out=b.out, lse=b.lse, **kw):
        with pytest.raises(ValueError, match=match):
            pcb.tree_attention(q, k, v, out, lse, **{**good, **kw})

    refused("lse", lse=b.lse.double())
    refused("lse", lse=b.lse[:-1])
    refused("lse", lse=b.lse.cpu())
    refused("lse", lse=torch.zeros((b.hq, b.n_rows), device="cuda").t())
    refused("out", out=b.out[:-1])
    refused("out", out=b.out.float())
    refused("q:", q=b.q.to(torch.float16))
    refused("q:", q=b.q.transpose(0, 1))
    refused("q:", q=torch.zeros((b.n_rows, b.hq, 64), dtype=torch.bfloat16, device="cuda"))
    refused("k:", k=b.k.float())
    refused("v:", v=b.v[:-16])
    refused("v:", v=b.v.to(torch.float16))
    refused("ctx_len", ctx_len=b.ctx_len.long())
    refused("row_start", row_start=b.row_start_d[:-1])
    refused("mask", mask=b.mask.int())
    refused("mask", mask=b.mask[:-1])
    refused("page_table", page_table=b.page_table[:1])
    refused("page_table", page_table=None)
    refused("page_table", ctx_start=b.ctx_len)
    refused("workspace", workspace=b.ws.int())
    w = torch.zeros((2, b.hkv, b.max_len), device="cuda")
    keep, count = torch.zeros((2, b.hkv, 8), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for match, call in (("weights_out", lambda: pcb.attention_weights(b.q, b.k, b.lse, w, w[:, :1], **good)),
                        ("use", lambda: pcb.attention_weights(b.q, b.k, b.lse, w, use=torch.zeros(1, dtype=torch.uint8, device="cuda"), **good)),
                        ("keep", lambda: pcb.select_slots(w, count, keep[:, :1], count)),
                        ("length", lambda: pcb.select_slots(w, count[:1], keep, count)),
                        ("count", lambda: pcb.select_slots(w, count, keep, count.float())),
                        ("keep", lambda: pcb.compact_slots(b.k, b.v, keep[:1], count, max_len=b.max_len, page_table=b.page_table)),
                        ("first", lambda: pcb.compact_slots(b.k, b.v, keep, count, max_len=b.max_len, page_table=b.page_table, first=count[:1]))):
        with pytest.raises(ValueError, match=match):
            call()
    with pytest.raises(TypeError):
        pcb.select_slots(w, count, keep, count, sink="1")
    with pytest.raises(ValueError):
        pcb.select_slots(w, count, keep, count, sink=2 ** 40)
    with pytest.raises(pcb.PerCacheError):
        pcb.select_slots(w, count, keep, count, sink=5, recent=4)


def test_a_batch_without_rows_only_decays_its_weights():
    b = Batch([(300, 0), (5, 0)], pad_rows=0)
    assert b.q.shape[0] == 0
    b.attend()
    w = torch.rand((2, b.hkv, b.max_len), device="cuda")
    before = w.clone()
    pcb.attention_weights(b.q, b.k, b.lse, w, decay=0.5, **b.args())
    check_weights(b, w, before, None, 0.5)


def test_two_calls_at_once_with_a_workspace_each():
    parts = [Batch([(6000, 9)], mask="tree", seed=1), Batch([(7000, 1), (100, 3)], seed=2, dtype="f16", paged=False)]
    streams = [torch.cuda.Stream() for _ in parts]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, s in zip(parts, streams):
            pcb.tree_attention(b.q, b.k, b.v, b.out, b.lse, **b.args(), stream=s.cuda_stream)
    torch.cuda.synchronize()
    for b in parts:
        pcb.ops_status(b.ws)
        b.check()


def test_one_workspace_for_all_calls_of_a_stream():
    parts = [Batch([(6000, 9)], mask="tree", seed=1), Batch([(7000, 1), (100, 3)], seed=2, dtype="f16", paged=False),
             Batch([(900, 40)], seed=3, mask="tree")]
    ws = parts[0].ws
    for b in parts:
        b.ws = ws
    for _ in range(10):
        for b in parts:
            pcb.tree_attention(b.q, b.k, b.v, b.out, b.lse, **b.args())
    for b in parts:
        b.check()


def test_captured_selection_and_moves_follow_their_arrays():
    n, h, budget = 700, 2, 64
    k, v = _pools(n, h, 128, "f16")
    k0, v0 = k.clone(), v.clone()
    w = torch.zeros((1, h, n), device="cuda")
    length = torch.tensor([n], dtype=torch.int32).cuda()
    start = torch.zeros(1, dtype=torch.int32, device="cuda")
    keep = torch.zeros((1, h, budget), dtype=torch.int32, device="cuda")
    count = torch.zeros(1, dtype=torch.int32, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            pcb.select_slots(w, length, keep, count, sink=1, recent=3, stream=side.cuda_stream)
            pcb.compact_slots(k, v, keep, count, max_len=n, weights=w, ctx_start=start, stream=side.cuda_stream)
    for m in (700, 65, 40):
        fresh = torch.rand((1, h, n), device="cuda")
        k.copy_(k0)
        v.copy_(v0)
        w.copy_(fresh)
        length.fill_(m)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for g in range(h):
            at = ops.select_slots(fresh[0, g].cpu().numpy(), m, budget, 1, 3)
            assert count.item() == len(at) and keep[0, g, :len(at)].tolist() == at
            assert torch.equal(k[:len(at), g].view(torch.int16), k0[at, g].view(torch.int16))
            assert torch.equal(v[len(at):, g].view(torch.int16), v0[len(at):, g].view(torch.int16))
            assert torch.equal(w[0, g, :len(at)], fresh[0, g, at])


def test_moves_to_another_place_take_any_list():
    k, v = _pools(128, 2, 64, "bf16")
    k0 = k.clone()
    keep = torch.tensor([[[9, 9, 3, 40, 0], [1, 63, 63, 2, 9]]], dtype=torch.int32).cuda()
    start, dst = torch.tensor([0], dtype=torch.int32).cuda(), torch.tensor([64], dtype=torch.int32).cuda()
    pcb.compact_slots(k, v, keep, torch.tensor([5], dtype=torch.int32).cuda(), max_len=64, ctx_start=start, dst_start=dst)
    for g in range(2):
        assert torch.equal(k[64:69, g].view(torch.int16), k0[keep[0, g].long(), g].view(torch.int16))
    assert torch.equal(k[:64].view(torch.int16), k0[:64].view(torch.int16))


@pytest.mark.parametrize("value", [0.0, 1.0, float("nan"), float("-inf")])
@pytest.mark.parametrize("n", [300, 20000])
def test_equal_weights_keep_the_lowest_slots(value, n):
    w = torch.full((1, 1, n), value, device="cuda")
    keep = torch.empty((1, 1, n // 2), dtype=torch.int32, device="cuda")
    count = torch.empty(1, dtype=torch.int32, device="cuda")
    pcb.select_slots(w, torch.tensor([n], dtype=torch.int32).cuda(), keep, count, sink=2, recent=5)
    want = list(range(n // 2 - 5)) + list(range(n - 5, n))
    assert keep[0, 0].tolist() == want and count.item() == n // 2


def test_a_run_of_steps_draft_verify_accept_evict():
    """The operators together, as a server uses them: a tree is verified, one path of it accepted and moved behind the
    context, its weights added, and the context cut to a budget; the next step attends to what is left."""
    b = Batch([(300, 7), (90, 7)], mask="tree", hq=4, hkv=2, dtype="f16")
    w = torch.zeros((2, 2, b.max_len), device="cuda")
    b.attend()
    b.check()
    # accept node 0 and the deepest node below it
    path = []
    for s in range(2):
        m = b.node_mask[s]
        deep = int(np.argmax(m.sum(1)))
        path.append(np.flatnonzero(m[deep]))
    use = torch.zeros(b.n_rows, dtype=torch.uint8, device="cuda")
    for s in range(2):
        use[torch.from_numpy(path[s] + int(b.row_start[s])).cuda()] = 1
    pcb.attention_weights(b.q, b.k, b.lse, w, use=use, **b.args())
    check_weights(b, w, torch.zeros_like(w), use.cpu().numpy(), 1.0)
    ctx = [c for c, _ in b.seqs]
    budget = max(len(p) for p in path)
    keep = torch.full((2, 1, budget), -1, dtype=torch.int32)
    for s in range(2):
        keep[s, 0, :len(path[s])] = torch.from_numpy((ctx[s] + path[s]).astype(np.int32))
    count = torch.tensor([len(p) for p in path], dtype=torch.int32)
    before = [(f64(b.k[torch.from_numpy(b.rows[s]).cuda()]), f64(b.v[torch.from_numpy(b.rows[s]).cuda()])) for s in range(2)]
    w_before = f64(w)
    pcb.compact_slots(b.k, b.v, keep.cuda(), count.cuda(), max_len=b.max_len, weights=w, first=b.ctx_len, page_table=b.page_table)
    length = (b.ctx_len + count.cuda()).to(torch.int32)
    keep2 = torch.empty((2, 2, 64), dtype=torch.int32, device="cuda")
    count2 = torch.empty(2, dtype=torch.int32, device="cuda")
    pcb.select_slots(w, length, keep2, count2, sink=2, recent=8, max_len=b.max_len)
    pcb.compact_slots(b.k, b.v, keep2, count2, max_len=b.max_len, weights=w, page_table=b.page_table)
    kept = keep2.cpu().numpy()
    for s in range(2):
        at = np.concatenate([np.arange(ctx[s]), ctx[s] + path[s]])
        for g in range(2):
            now = ops.select_slots(w_before[s, g, at].astype(np.float32), len(at), 64, 2, 8)
            assert kept[s, g].tolist() == now
            rows = torch.from_numpy(b.rows[s][:64]).cuda()
            assert np.array_equal(f64(b.k[rows, g]), before[s][0][at[now], g])
            assert np.array_equal(f64(b.v[rows, g]), before[s][1][at[now], g])
            assert np.array_equal(f64(w[s, g, :64]), w_before[s, g, at[now]])
    # the next tokens, on the 64 slots that are left
    c = Batch([(64, 3), (64, 3)], hq=4, hkv=2, dtype="f16", seed=9)
    for s in range(2):
        own = torch.from_numpy(b.rows[s][:67]).cuda()
        c.rows[s] = b.rows[s][:67]
        b.k[own[64:]] = c.k[:3]
        b.v[own[64:]] = c.v[:3]
        b.k[own[64:]] = torch.randn((3, 2, 128), device="cuda").half()
        b.v[own[64:]] = torch.randn((3, 2, 128), device="cuda").half()
    c.k, c.v, c.page_table, c.max_len = b.k, b.v, b.page_table, b.max_len
    c.attend()
    c.check()
