"""Operators that write, read and share a decoding batch's pages, against the float64 oracle.

Tolerances.  append_rows: the norm is a sum of D squares, a reciprocal root and two products in fp32, the rotation two products and a sum of
values no larger than the pair's length: off by at most (D + 12) * 2^-24 of that length (2^-16 of the head's largest |value| covers it, with the
gain's spread), then half a step of the stored type.  Without norm and rotation the 8-bit bytes are the oracle's, bit for bit.
tree_attention_8bit: a score is a sum of D products, exact in 8 bits, accumulated with an error of at most D * 2^-23 of the sum of magnitudes (measured
2^-21), of q's parts: the row's largest counts 224 or more there, the last part's least step is 2^-9 and it counts 2^-4 (two parts: bf16) of
that, so half a step, what they leave of an element, is 2^-10 * 2^-4 / 224 < 2^-21 of the row's largest |q| (fp16's third part: less); weights are split
to half a step of the 16-bit type or finer, with an absolute floor of 2^-32 of the row's largest (2^16 slots: 2^-16 of the largest |v|), the output is rounded once.
"""
import numpy as np
import pytest

from oracle import cache_ops as ops
from oracle import pages as P
from paper_2601_11553_b200 import percache as pcb

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
F8 = torch.float8_e4m3fn


def f64(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def raw(pages):
    return pages.view(torch.uint8).cpu().numpy()


def table_of(lens, rng, width, spare=2):
    """Shuffled page ids; entries that are never used point nowhere."""
    pages = [-(-x // 16) for x in lens]
    order = rng.permutation(sum(pages) + spare)
    table = np.full((len(lens), width), 10 ** 6, dtype=np.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = order[at:at + p]
        at += p
    return table, len(order)


# ---------------------------------------------------------------------------------------------------------------- attention
class Batch:
    def __init__(self, seqs, dtype="bf16", hq=4, hkv=2, d=128, mask=None, seed=0, q_scale=1.0, pad_rows=3, wide=0, layers=1, scale_spread=3, pow2=True):
        self.seqs, self.hq, self.hkv, self.d = seqs, hq, hkv, d
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        t = TYPES[dtype]
        lens = [c + n for c, n in seqs]
        self.max_len = max(max(lens, default=1), 1)
        self.max_nodes = max(max((n for _, n in seqs), default=1), 1)
        self.table, total = table_of(lens, rng, -(-self.max_len // 16))
        # every byte that no prompt owns, and every scale of such a page, is NaN
        big = torch.full((total, layers, hkv, 2, 16, d), 0x7f, dtype=torch.uint8, device="cuda")
        self.pages = big[:, layers - 1].view(F8)
        self.scales = torch.full((total, hkv, 2), float("nan"), device="cuda")
        for b, n in enumerate(lens):
            ids = torch.from_numpy(self.table[b, :-(-n // 16)].astype(np.int64)).cuda()
            if n == 0:
                continue
            x = (100 * torch.randn((len(ids), hkv, 2, 16, d), generator=gen, device="cuda")).clamp(-448, 448).to(F8).view(torch.uint8)
            if n % 16:
                x[-1, :, :, n % 16:] = 0x7f
            self.pages.view(torch.uint8)[ids] = x
            e = torch.randint(-7 - scale_spread, -6, (len(ids), hkv, 2), generator=gen, device="cuda").float()
            self.scales[ids] = torch.exp2(e) * (1 if pow2 else 1 + torch.rand(e.shape, generator=gen, device="cuda"))
        self.row_start = np.concatenate([[0], np.cumsum([n for _, n in seqs])]).astype(np.int32)
        self.n = int(self.row_start[-1])
        self.n_rows = self.n + pad_rows
        q = (q_scale * torch.randn((self.n_rows, hq * d + wide), generator=gen, device="cuda")).to(t)
        self.q = q.as_strided((self.n_rows, hq, d), (hq * d + wide, d, 1))
        self.out = torch.full((self.n_rows, hq * d + wide), 7.0, dtype=t, device="cuda").as_strided((self.n_rows, hq, d), (hq * d + wide, d, 1))
        self.lse = torch.full((self.n_rows, hq), 7.0, device="cuda")
        self.node_mask, self.mask = [None] * len(seqs), None
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
                    for j in list(np.flatnonzero(m[i])) + list(range(n, 64 * words)):      # bits past the prompt's nodes mean nothing
                        bits[self.row_start[b] + i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
            self.mask = torch.from_numpy(bits.view(np.int64)).cuda()
        self.page_table, self.ctx_len, self.row_start_d = torch.from_numpy(self.table).cuda(), i32([c for c, _ in seqs]), torch.from_numpy(self.row_start).cuda()
        self.ws = torch.zeros(pcb.OPS_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
        self.scale = d ** -0.5

    def attend(self, **kw):
        pcb.tree_attention_8bit(self.q, self.pages, self.scales, self.out, self.lse,
                                **{**dict(ctx_len=self.ctx_len, row_start=self.row_start_d, page_table=self.page_table, mask=self.mask,
                                          max_nodes=self.max_nodes, max_len=self.max_len, scale=self.scale, workspace=self.ws), **kw})
        pcb.ops_status(self.ws)

    def kv(self, b, length):
        """Keys and values [slots, hkv, d] of a prompt."""
        ids = self.table[b, :-(-length // 16)].astype(np.int64)
        own = (ids >= 0) & (ids < len(self.pages))
        at = torch.from_numpy(np.where(own, ids, 0)).cuda()
        x = P.VALUES[raw(self.pages[at])] * f64(self.scales[at]).clip(2.0 ** -32, 2.0 ** 32)[..., None, None]
        x[~own] = 0
        x = x.transpose(2, 0, 3, 1, 4).reshape(2, -1, self.hkv, self.d)[:, :length]
        return x[0], x[1]

    def check(self):
        q, out, lse = f64(self.q), f64(self.out), f64(self.lse)
        eps = torch.finfo(self.q.dtype).eps / 2
        for b, (c, n) in enumerate(self.seqs):
            if n == 0:
                continue
            r0, r1 = int(self.row_start[b]), int(self.row_start[b + 1])
            k, v = self.kv(b, c + n)
            want, wlse, mean_abs = ops.tree_attention(q[r0:r1], k, v, c, self.node_mask[b], self.scale)
            delta = self.delta(q[r0:r1], k, ops.sees(n, c, self.node_mask[b]))
            vmax = np.abs(v[np.isfinite(v)]).max(initial=0.0)
            tol = (eps + 2 * delta[:, :, None] + 2.0 ** -18) * mean_abs + eps * np.abs(want) + 2.0 ** -16 * vmax + 1e-30
            assert np.array_equal(np.isnan(out[r0:r1]), np.isnan(want)), b
            fine = np.isfinite(want)
            diff = np.abs(out[r0:r1] - want)
            assert (diff[fine] <= tol[fine]).all(), (b, c, n, diff[fine].max(), int((diff[fine] > tol[fine]).sum()), fine.sum())
            assert np.array_equal(np.isnan(lse[r0:r1]), np.isnan(wlse))
            lf = np.isfinite(wlse)
            assert np.array_equal(lse[r0:r1][~lf & ~np.isnan(wlse)], wlse[~lf & ~np.isnan(wlse)])
            ltol = delta + 2.0 ** -20 * (np.abs(np.where(lf, wlse, 0)) + 4)
            assert (np.abs(lse[r0:r1] - wlse)[lf] <= ltol[lf]).all(), (b, np.abs(lse[r0:r1] - wlse)[lf].max())
        assert (out[self.n:] == 7.0).all() and (lse[self.n:] == 7.0).all()

    def delta(self, q, k, seen):
        group = self.hq // self.hkv
        kk = np.abs(np.repeat(np.nan_to_num(k), group, axis=1))
        with np.errstate(invalid="ignore", over="ignore"):
            x = np.einsum("nhd,thd->nht", np.abs(q), kk) * self.d * 2.0 ** -23
            x += np.abs(q).max(-1)[:, :, None] * kk.sum(-1).T[None] * 2.0 ** -21
        x = np.where(np.isfinite(x) & seen[:, None, :], x * self.scale, 0)
        return x.max(axis=2, initial=0.0)


SHAPES = [
    # one token, at lengths around the page and block borders
    dict(seqs=[(0, 1)]), dict(seqs=[(1, 1)], dtype="f16"), dict(seqs=[(15, 1)]), dict(seqs=[(16, 1)], d=64), dict(seqs=[(126, 1)]), dict(seqs=[(127, 1)], dtype="f16"),
    dict(seqs=[(128, 1)]), dict(seqs=[(255, 1)], d=64, dtype="f16"), dict(seqs=[(256, 1)]), dict(seqs=[(767, 1)]), dict(seqs=[(768, 1)], dtype="f16"),
    dict(seqs=[(1000, 1)], hq=16, hkv=8),
    # head layouts: one to 128 query heads a KV head, tiles that end inside a node's heads
    dict(seqs=[(200, 3)], hq=1, hkv=1), dict(seqs=[(200, 3)], hq=3, hkv=1, mask="tree"), dict(seqs=[(200, 7)], hq=14, hkv=2, dtype="f16", mask="tree"),
    dict(seqs=[(77, 9)], hq=128, hkv=1, mask="tree"), dict(seqs=[(300, 2)], hq=100, hkv=2, d=64), dict(seqs=[(1300, 11)], hq=12, hkv=1, mask="tree", dtype="f16"),
    # trees: around the word and tile borders, up to the most nodes
    dict(seqs=[(100, 8)], mask="tree"), dict(seqs=[(100, 9)], mask="tree"), dict(seqs=[(100, 64)], mask="tree", dtype="f16"), dict(seqs=[(100, 65)], mask="tree"),
    dict(seqs=[(333, 256)], mask="tree", dtype="f16"), dict(seqs=[(0, 256)], mask="tree"), dict(seqs=[(5, 200)], mask="random", d=64), dict(seqs=[(640, 130)], hq=6),
    dict(seqs=[(0, 17)]), dict(seqs=[(0, 40)], mask="empty"), dict(seqs=[(3, 40)], mask="empty"), dict(seqs=[(0, 70)], mask="random", dtype="f16"),
    # ragged batches, prompts without nodes and without context among them
    dict(seqs=[(700, 1), (3, 12), (0, 1), (129, 30), (64, 0), (2000, 7)], mask="tree"),
    dict(seqs=[(700, 1), (3, 12), (0, 0), (129, 30), (64, 0), (2000, 7)], mask="tree", dtype="f16", hq=8, d=64),
    dict(seqs=[(i % 37, 1 + i % 3) for i in range(300)], hq=2, hkv=1, mask="tree"), dict(seqs=[(1500 + 131 * i, 1) for i in range(9)], hq=16, hkv=8, dtype="f16"),
    # long contexts: split over many blocks
    dict(seqs=[(20000, 1)], hq=2, hkv=1), dict(seqs=[(33024, 4)], hq=4, hkv=1, dtype="f16"), dict(seqs=[(9000, 48)], mask="tree"),
    # rows further apart than their heads need, pages of one layer among others
    dict(seqs=[(300, 6), (40, 2)], wide=8, mask="tree", layers=3), dict(seqs=[(300, 6), (40, 2)], wide=136, dtype="f16", d=64, layers=2),
    # large scores; scales far apart; scales that are no powers of two
    dict(seqs=[(400, 20)], q_scale=12.0, mask="tree"), dict(seqs=[(1200, 3)], q_scale=30.0, dtype="f16"), dict(seqs=[(900, 5)], scale_spread=14),
    dict(seqs=[(900, 5)], scale_spread=14, dtype="f16"), dict(seqs=[(900, 5)], pow2=False), dict(seqs=[(900, 5)], pow2=False, dtype="f16"),
]


@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_attention_matches_the_oracle(case):
    b = Batch(seed=case, **SHAPES[case])
    b.attend()
    b.check()


def test_attention_without_lse_and_the_same_every_time():
    b = Batch([(5000, 9), (130, 2), (0, 1)], mask="tree", hq=8)
    b.attend()
    first = b.out.clone()
    for _ in range(3):
        b.out.fill_(7.0)
        pcb.tree_attention_8bit(b.q, b.pages, b.scales, b.out, ctx_len=b.ctx_len, row_start=b.row_start_d, page_table=b.page_table, mask=b.mask,
                                max_nodes=b.max_nodes, max_len=b.max_len, workspace=b.ws)
        assert torch.equal(first, b.out)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_many_slots_under_a_heavy_one_are_not_lost(dtype):
    """One slot has nearly all weight and values near zero: the result is what the 30000 others add."""
    b = Batch([(30000, 1)], dtype=dtype, hq=2, hkv=1, q_scale=0.01)
    page = int(b.table[0, 0])
    b.pages.view(torch.uint8)[page, 0, 0, 0] = 0x7e                          # the key of slot 0: 448 in every element
    b.pages.view(torch.uint8)[page, 0, 1, 0] = 0
    b.q[0] = 0.26 if dtype == "f16" else 0.25
    b.scales[page, 0, 0] = 2.0 ** -6
    b.attend()
    q, out = f64(b.q), f64(b.out)
    k, v = b.kv(0, 30001)
    want, _, mean_abs = ops.tree_attention(q[:1], k, v, 30000, None, b.scale)
    x = ops.scores(q[:1], k, b.scale)
    assert ((x.max(-1) - np.median(x, -1)) * np.log2(np.e) > 16).all()       # the others weigh less than 2^-16 of it each
    delta = b.delta(q[:1], k, ops.sees(1, 30000, None))[:, :, None]
    eps = torch.finfo(b.q.dtype).eps / 2
    assert (np.abs(out[:1] - want) <= (eps + 2 * delta + 2.0 ** -18) * mean_abs + eps * np.abs(want) + 30000 * 2.0 ** -32 * np.abs(v).max()).all()


def test_nan_and_infinity_reach_who_sees_them_only():
    b = Batch([(140, 6), (50, 3)], mask="tree", seed=4)
    page = int(b.table[0, 142 // 16])
    b.pages.view(torch.uint8)[page, :, 1, 142 % 16, 5] = 0xff                # node 2's value
    b.pages.view(torch.uint8)[page, 0, 0, 143 % 16, 9] = 0x7f                # node 3's key, first KV head
    b.attend()
    b.check()
    assert np.isnan(f64(b.out[2, :, 5])).all() and np.isfinite(f64(b.out[0])).all()
    b = Batch([(140, 6), (50, 3)], seed=5, dtype="f16")
    b.q[1, 0, 3], b.q[7, 3, 0] = float("inf"), float("nan")
    b.attend()
    out = f64(b.out)
    assert np.isnan(out[1, 0]).all() and np.isnan(out[7, 3]).all()
    out[1, 0] = out[7, 3] = 0
    assert np.isfinite(out[:9]).all()


def test_nan_in_the_context_reaches_every_row_of_its_head():
    b = Batch([(300, 2)], seed=6)
    b.pages.view(torch.uint8)[int(b.table[0, 3]), 1, 1, 4, 77] = 0x7f
    b.attend()
    b.check()
    assert np.isnan(f64(b.out)[:2, 2:, 77]).all() and np.isfinite(f64(b.out)[:2, :2]).all()


def test_pages_outside_the_pool_hold_zeros():
    b = Batch([(400, 2), (64, 1)], seed=7)
    b.table[0, 2], b.table[0, 9], b.table[1, 0] = -1, 10 ** 9, len(b.pages)
    b.page_table.copy_(torch.from_numpy(b.table))
    b.attend()
    b.check()


def test_scales_outside_the_range_count_as_its_ends():
    b = Batch([(100, 2)], seed=8)
    b.scales[int(b.table[0, 1]), :, 0] = 0.0
    b.scales[int(b.table[0, 2]), :, 1] = 2.0 ** -40
    b.scales[int(b.table[0, 3]), 0, 1] = 2.0 ** 32
    b.attend()
    b.check()


def test_empty_calls_write_nothing():
    b = Batch([(30, 0), (0, 0)])
    b.attend()
    assert (b.out == 7).all() and (b.lse == 7).all()
    b = Batch([], pad_rows=2)
    b.attend()
    assert (b.out == 7).all()


def test_attention_on_another_stream_and_replayed_with_new_lengths():
    b = Batch([(900, 3), (200, 1)], seed=9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.attend()
    s.synchronize()
    b.check()
    g = torch.cuda.CUDAGraph()
    args = dict(ctx_len=b.ctx_len, row_start=b.row_start_d, page_table=b.page_table, max_nodes=b.max_nodes, max_len=b.max_len, scale=b.scale, workspace=b.ws)
    with torch.cuda.graph(g):
        pcb.tree_attention_8bit(b.q, b.pages, b.scales, b.out, b.lse, **args)
        pcb.tree_attention_8bit(b.q, b.pages, b.scales, b.out, b.lse, **args)
    for seqs in ([(900, 3), (200, 1)], [(640, 1), (100, 3)], [(0, 2), (199, 2)]):
        # slots behind the new ends are left in use: the rows there hold finite values, or NaN that nobody may see
        b.seqs = seqs
        b.row_start = np.concatenate([[0], np.cumsum([n for _, n in seqs])]).astype(np.int32)
        b.n = int(b.row_start[-1])
        b.ctx_len.copy_(i32([c for c, _ in seqs])), b.row_start_d.copy_(torch.from_numpy(b.row_start))
        b.out.fill_(7.0), b.lse.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        b.check()


# ---------------------------------------------------------------------------------------------------------------- append
class Rows:
    """New rows of a batch; seqs: [(slots in use, new rows)]."""

    def __init__(self, seqs, dtype="bf16", hq=4, hkv=2, d=128, cache="8bit", norm=True, rope=True, position=False, seed=0, pad_rows=2, spread=1.0, packed=True):
        self.seqs, self.hq, self.hkv, self.d, self.cache = seqs, hq, hkv, d, cache
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        t = TYPES[dtype]
        lens = [c + n for c, n in seqs]
        self.max_len = max(max(lens, default=1), 1)
        self.row_start = np.concatenate([[0], np.cumsum([n for _, n in seqs])]).astype(np.int32)
        self.n = int(self.row_start[-1])
        rows = self.n + pad_rows
        x = torch.randn((rows, hq + 2 * hkv, d), generator=gen, device="cuda") * torch.exp2(spread * torch.randn((rows, 1, 1), generator=gen, device="cuda"))
        x = x.to(t)
        self.q, self.k, self.v = (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]) if packed else (x[:, :hq].contiguous(), x[:, hq:hq + hkv].contiguous(), x[:, hq + hkv:].contiguous())
        self.q_out = torch.full((rows, hq, d), 7.0, dtype=t, device="cuda")
        self.kw = dict(ctx_len=i32([c for c, _ in seqs]), row_start=torch.from_numpy(self.row_start).cuda(), max_len=self.max_len, eps=1e-5)
        self.gains = [None, None]
        if norm:
            self.gains = [1 + 0.3 * torch.randn(d, generator=gen, device="cuda") for _ in range(2)]
            self.kw.update(q_gain=self.gains[0], k_gain=self.gains[1])
        self.rope, self.position = None, None
        if rope:
            n_pos = 2 * self.max_len + 7
            angle = np.arange(n_pos)[:, None] * 1e6 ** (-np.arange(d // 2) / (d // 2))
            self.rope = torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)).cuda()
            self.kw["rope"] = self.rope
            if position:
                self.position = rng.integers(-2, n_pos + 3, rows).astype(np.int32)               # outside the table too: clamped
                self.kw["position"] = torch.from_numpy(self.position).cuda()
        self.table = None
        if cache != "slots":
            self.table, total = table_of(lens, rng, -(-self.max_len // 16))
            self.kw["page_table"] = torch.from_numpy(self.table).cuda()
        else:
            self.start = np.cumsum([3] + [x + 2 for x in lens])[:-1].astype(np.int32)
            self.kw["ctx_start"] = torch.from_numpy(self.start).cuda()
            total = -(-(3 + sum(lens) + 2 * len(lens)) // 16)
        if cache == "8bit":
            self.pages = torch.randint(0, 0x7f, (total, hkv, 2, 16, d), generator=gen, device="cuda", dtype=torch.uint8).view(F8)
            self.scales = torch.exp2(torch.randint(-14, 1, (total, hkv, 2), generator=gen, device="cuda").float())
            self.kw.update(pages=self.pages, scales=self.scales)
            self.before = raw(self.pages).copy(), self.scales.cpu().numpy().copy()
        else:
            self.pool = [torch.randn((total * 16, hkv, d), generator=gen, device="cuda").to(t) for _ in range(2)]
            self.kw.update(k_pool=self.pool[0], v_pool=self.pool[1])
            self.before = [f64(p) for p in self.pool]

    def run(self, q=True, **kw):
        pcb.append_rows(self.q if q else None, self.k, self.v, self.q_out if q else None, **{**self.kw, **kw})
        torch.cuda.synchronize()

    def wanted(self):
        """Per prompt: the rows' queries, keys and values before their rounding."""
        for b, (c, n) in enumerate(self.seqs):
            r = slice(int(self.row_start[b]), int(self.row_start[b + 1]))
            t = None
            if self.rope is not None:
                pos = np.arange(c, c + n) if self.position is None else self.position[r].clip(0, len(self.rope) - 1)
                t = f64(self.rope)[pos]
            gq, gk = (None if g is None else f64(g) for g in self.gains)
            yield b, c, n, r, P.norm_rotate(f64(self.q[r]), gq, 1e-5, t), P.norm_rotate(f64(self.k[r]), gk, 1e-5, t), f64(self.v[r])

    def arith(self, x):
        """What fp32 arithmetic may be off by."""
        exact = self.rope is None and self.gains[0] is None
        return np.zeros(x.shape) if exact else 2.0 ** -16 * np.abs(x).max(-1, keepdims=True)

    def near(self, got, want, half_step, name):
        fine = np.isfinite(want)
        assert np.array_equal(np.isfinite(got), fine), name
        tol = np.abs(np.where(fine, want, 0)) * half_step + self.arith(np.where(fine, want, 0)) * (1 + half_step) + 2.0 ** -25
        assert (np.abs(got - want)[fine] <= tol[fine]).all(), (name, np.abs(got - want)[fine].max())

    def check(self, q=True):
        eps = torch.finfo(self.q.dtype).eps / 2
        got_q = f64(self.q_out)
        if self.cache == "8bit":
            now, now_s = raw(self.pages), self.scales.cpu().numpy()
            touched = np.zeros(now.shape[:1] + (16,), dtype=bool)
            fresh = np.zeros(now.shape[:1], dtype=bool)
        else:
            got, wrote = [f64(p) for p in self.pool], np.zeros(len(self.pool[0]), dtype=bool)
        for b, c, n, r, wq, wk, wv in self.wanted():
            if q:
                self.near(got_q[r], wq, eps, "q")
            if self.cache != "8bit":
                slots = np.arange(c, c + n)
                at = self.table[b, slots // 16].astype(np.int64) * 16 + slots % 16 if self.table is not None else slots + self.start[b]
                self.near(got[0][at], wk, eps, "k")
                assert np.array_equal(got[1][at], wv)
                wrote[at] = True
                continue
            for j in range(c // 16, -(-(c + n) // 16) if n else c // 16):
                lo, hi, page = max(16 * j, c), min(16 * j + 16, c + n), self.table[b, j]
                touched[page, :hi - 16 * j] = True
                fresh[page] = True
                for h in range(self.hkv):
                    for w, x in enumerate((wk, wv)):
                        new = x[lo - c:hi - c, h]
                        want, s = P.fill_page(self.before[0][page, h, w], float(self.before[1][page, h, w]), lo - 16 * j, new)
                        got8, got_s = now[page, h, w], float(now_s[page, h, w])
                        if got_s != s:         # the largest value is within the arithmetic's error of a border
                            amax = np.abs(new).max()
                            e = np.log2(min(s, got_s) * 448 / amax)
                            assert w == 0 and self.arith(new).max() > 0 and max(s, got_s) == 2 * min(s, got_s) and abs(e) < 2.0 ** -14, (s, got_s, amax)
                            continue
                        a, z = lo - 16 * j, hi - 16 * j
                        assert np.array_equal(got8[:a] & 0x7f, want[:a] & 0x7f) and np.array_equal(got8[z:], want[z:])
                        if w == 1 or self.arith(new).max() == 0:
                            assert np.array_equal(got8[:z], want[:z])
                        else:
                            err = np.abs(P.VALUES[got8[a:z]] * s - new)
                            assert (err <= np.maximum(np.abs(new) * 2.0 ** -4, s * 2.0 ** -10) + self.arith(new) * (1 + 2.0 ** -4)).all()
        if self.cache == "8bit":
            keep = np.broadcast_to(~touched[:, None, None, :, None], now.shape)
            assert np.array_equal(now[keep], self.before[0][keep]) and np.array_equal(now_s[~fresh], self.before[1][~fresh])
        else:
            for x, y in zip(got, self.before):
                assert np.array_equal(x[~wrote], y[~wrote])
        assert (got_q[self.n:] == 7).all() and (q or (got_q == 7).all())


APPENDS = [
    dict(seqs=[(0, 1)]), dict(seqs=[(5, 1)]), dict(seqs=[(15, 1)]), dict(seqs=[(16, 1)]), dict(seqs=[(0, 16)]), dict(seqs=[(0, 17)]), dict(seqs=[(9, 40)]),
    dict(seqs=[(31, 2)]), dict(seqs=[(3, 5)]), dict(seqs=[(100, 333)], hq=16, hkv=8),
    dict(seqs=[(17, 3), (0, 0), (40, 1), (0, 64), (15, 18), (7, 0)]), dict(seqs=[(i % 53, 1) for i in range(200)], hq=2, hkv=1),
    dict(seqs=[(i % 21, i % 4) for i in range(700)], hq=1, hkv=1), dict(seqs=[(0, 3000)], hq=2, hkv=1), dict(seqs=[(2, 700), (333, 900)], hq=6, hkv=3),
    dict(seqs=[(20, 30)], hq=12, hkv=4), dict(seqs=[(5, 9)], hq=7, hkv=1), dict(seqs=[(5, 9)], hq=33, hkv=11),
]


@pytest.mark.parametrize("case", range(len(APPENDS)))
@pytest.mark.parametrize("kind", [dict(cache="8bit"), dict(cache="8bit", d=64, dtype="f16", position=True), dict(cache="pages", dtype="f16"),
                                  dict(cache="slots", d=64, position=True), dict(cache="8bit", norm=False, rope=False, dtype="f16"),
                                  dict(cache="8bit", norm=False, rope=False, d=64, packed=False), dict(cache="pages", norm=False, packed=False),
                                  dict(cache="slots", rope=False, dtype="f16")], ids=str)
def test_append_matches_the_oracle(case, kind):
    r = Rows(seed=case, **{**APPENDS[case], **kind})
    r.run()
    r.check()


@pytest.mark.parametrize("cache", ["8bit", "pages"])
def test_append_without_queries_and_with_queries_in_place(cache):
    r = Rows([(3, 20), (40, 1)], cache=cache)
    r.run(q=False)
    r.check(q=False)
    r = Rows([(3, 20), (40, 1)], cache=cache, packed=False)
    q = r.q.clone()
    pcb.append_rows(q, r.k, r.v, q, **r.kw)
    r.q_out[:r.n] = q[:r.n]
    assert torch.equal(q[r.n:], r.q[r.n:])
    r.check()


def test_only_queries_or_only_keys_are_normalised():
    for which in (0, 1):
        r = Rows([(3, 20)], hq=5, hkv=3)
        r.gains[which] = None
        r.kw["q_gain" if which == 0 else "k_gain"] = None
        r.run()
        r.check()


def test_large_small_and_odd_values():
    r = Rows([(0, 16), (3, 5)], norm=False, rope=False, cache="8bit")
    r.k[0, 0, 3], r.k[1, 0, 5], r.k[2, 1, 7] = float("inf"), float("-inf"), float("nan")
    r.v[4, 0], r.v[5, 1] = 0.0, 3e38
    r.v[16:21, 0] = 0.0                                       # zeros behind slots in use: the page's scale stays
    r.run()
    r.check()
    s = f64(r.scales)[r.table[0, 0]]
    assert s[1, 1] == 2.0 ** 32
    k = raw(r.pages)[r.table[0, 0]][:, 0]
    assert k[0, 0, 3] == 0x7e and k[0, 1, 5] == 0xfe and k[1, 2, 7] & 0x7f == 0x7f
    r = Rows([(0, 5)], norm=False, rope=False, cache="8bit")
    r.k.zero_()
    r.run()
    r.check()
    assert (f64(r.scales)[r.table[0, 0], :, 0] == 2.0 ** -32).all()


def test_fp16_saturates_and_nan_stays():
    r = Rows([(0, 3)], dtype="f16", cache="slots", norm=False)
    r.k[:] = 60000.0
    r.k[1, 0, 0], r.k[2, 0, 0] = float("inf"), float("nan")
    r.run()
    k = f64(r.pool[0])[r.start[0]:r.start[0] + 3]
    assert np.isnan(k[2, 0, 0]) and np.isnan(k[2, 0, 64]) and not np.isfinite(k[1, 0, 0])
    assert np.nanmax(np.abs(k[0])) <= 65504 and np.isfinite(k[0]).all()


def test_pages_and_slots_outside_the_pools_are_not_written():
    for cache in ("8bit", "pages", "slots"):
        r = Rows([(3, 40), (20, 30)], cache=cache)
        if cache == "slots":
            r.kw["ctx_start"] = i32([-100, 10 ** 6])
        else:
            bad = r.table.copy()
            bad[:, :] = -1
            bad[1] = 10 ** 8
            r.kw["page_table"] = torch.from_numpy(bad).cuda()
        r.run()
        if cache == "8bit":
            assert np.array_equal(raw(r.pages), r.before[0])
        else:
            assert all(np.array_equal(f64(x), y) for x, y in zip(r.pool, r.before))
        eps = torch.finfo(r.q.dtype).eps / 2
        for b, c, n, rr, wq, wk, wv in r.wanted():
            r.near(f64(r.q_out)[rr], wq, eps, "q")


def test_token_by_token_gives_what_the_prompt_gives_where_scales_agree():
    """Values within a factor of two of each other in every page: the page's scale does not depend on the order."""
    r = Rows([(0, 50)], norm=False, rope=False, spread=0.0)
    r.v.copy_(r.v.sign() * (1 + r.v.abs() % 1) * 0.75)
    r.k.copy_(r.k.sign() * (1 + r.k.abs() % 1) * 0.75)
    r.v[:, :, 0] = r.k[:, :, 0] = 1.5
    r.run()
    whole, scales = raw(r.pages).copy(), r.scales.clone()
    ids = r.table[0]
    r.pages.view(torch.uint8)[torch.from_numpy(ids.astype(np.int64)).cuda()] = 0x11
    for i in range(50):
        pcb.append_rows(None, r.k[i:i + 1], r.v[i:i + 1], **{**r.kw, "ctx_len": i32([i]), "row_start": i32([0, 1])})
    torch.cuda.synchronize()
    now = raw(r.pages)
    assert np.array_equal(now[ids[:3]], whole[ids[:3]]) and np.array_equal(now[ids[3], :, :, :2], whole[ids[3], :, :, :2])
    assert torch.equal(r.scales, scales)


def test_append_is_captured_and_replayed_on_another_batch():
    r = Rows([(30, 1), (5, 3), (0, 2)], seed=3)
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            pcb.append_rows(r.q, r.k, r.v, r.q_out, **r.kw)
    for seqs in ([(30, 1), (5, 3), (0, 2)], [(17, 2), (6, 0), (0, 1)]):
        r.seqs = seqs
        r.row_start = np.concatenate([[0], np.cumsum([n for _, n in seqs])]).astype(np.int32)
        r.n = int(r.row_start[-1])
        r.kw["ctx_len"].copy_(i32([c for c, _ in seqs])), r.kw["row_start"].copy_(torch.from_numpy(r.row_start))
        r.q_out.fill_(7.0)
        r.before = raw(r.pages).copy(), r.scales.cpu().numpy().copy()
        g.replay()
        torch.cuda.synchronize()
        r.check()


# ---------------------------------------------------------------------------------------------------------------- fork
class Forest:
    """Sequences that share pages, their counters and free list, and pools whose pages can be told apart."""

    def __init__(self, lengths, shared=0, spare=40, extra_held=0, seed=0, layers=2, width=None, pool_kinds=("f8", "scale")):
        rng = np.random.default_rng(seed)
        n = len(lengths)
        held = [-(-x // 16) + extra_held for x in lengths]
        total = shared + sum(h - shared for h in held) + spare
        order = list(rng.permutation(total))
        self.width = width or max(held, default=1) + 3
        self.table = [[-1] * self.width for _ in range(n)]
        common = [order.pop() for _ in range(shared)]
        for s in range(n):
            self.table[s][:held[s]] = common + [order.pop() for _ in range(held[s] - shared)]
        self.refs = [0] * total
        for s in range(n):
            for p in self.table[s][:held[s]]:
                self.refs[p] += 1
        self.free, self.held, self.length, self.total = [int(p) for p in order], held, list(lengths), total
        shapes = {"f8": ((layers, total, 3, 2, 16, 64), torch.uint8), "scale": ((layers, total, 3, 2), torch.float32), "bf16": ((layers, total, 16, 3, 64), torch.bfloat16),
                  "odd": ((1, total, 5), torch.int32), "big": ((1, total, 9000), torch.int32)}
        self.pools = [torch.randint(0, 120, shapes[k][0], device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(shapes[k][1]) for k in pool_kinds]
        self.ws = torch.randint(0, 255, (pcb.OPS_WORKSPACE_BYTES,), dtype=torch.uint8, device="cuda")        # another operator's leavings

    def fork(self, parent, room=1, width_out=None, in_place=False, run=True):
        width_out = width_out or self.width
        n, m = len(self.held), len(parent)
        listed = self.free + [-7] * (self.total - len(self.free))
        t = dict(page_table=i32(self.table).reshape(n, self.width), held=i32(self.held), length=i32(self.length), parent=i32(parent),
                 table_out=torch.full((m, width_out), 77, dtype=torch.int32, device="cuda"), held_out=i32([77] * m), length_out=i32([77] * m),
                 refs=i32(self.refs), free_list=i32(listed), free_count=i32([len(self.free)]), missing=i32([77]))
        outs = {} if in_place else dict(refs_out=i32([77] * self.total), free_list_out=i32([77] * self.total), free_count_out=i32([77]))
        before = [p.clone() for p in self.pools]
        pcb.fork_pages(**t, pools=self.pools, room=room, workspace=self.ws, **outs)
        torch.cuda.synchronize()
        table, held, length, refs, free, missing, copies = P.fork(self.table, self.held, self.length, parent, width_out, self.refs, self.free, room, self.total)
        got = {k: outs.get(k + "_out", t[k]).cpu().numpy().tolist() for k in ("refs", "free_list", "free_count")}
        want = [row + [-1] * (width_out - len(row)) for row in table]
        assert t["table_out"].cpu().numpy().tolist() == want
        assert t["held_out"].cpu().numpy().tolist() == held and t["length_out"].cpu().numpy().tolist() == length
        assert t["missing"].item() == missing and got["refs"] == refs
        assert got["free_count"] == [len(free)] and got["free_list"][:len(free)] == free
        assert got["free_list"][len(free):] == listed[len(free):] or len(free) < len(self.free)
        if not in_place:
            assert t["refs"].cpu().tolist() == self.refs and t["free_list"].cpu().tolist() == listed and t["free_count"].item() == len(self.free)
        for p, old in zip(self.pools, before):
            for a, b in copies:
                old[:, b] = old[:, a]
            assert torch.equal(p, old)
        self.table, self.held, self.length, self.refs, self.free, self.width = want, held, length, refs, free, width_out


FORKS = [
    dict(lengths=[37], parent=[0, 0, 0, 0]), dict(lengths=[48], parent=[0, 0]), dict(lengths=[48], parent=[0, 0], room=0), dict(lengths=[1], parent=[0]),
    dict(lengths=[0], parent=[0, 0, 0]), dict(lengths=[33, 40, 50], parent=[2, 0, 2, 2], shared=1), dict(lengths=[33, 40, 50], parent=[1, 1, 1], shared=2, room=40),
    dict(lengths=[100, 90, 80], parent=[], shared=5), dict(lengths=[100, 90, 80], parent=[-1, 3, 1, 99], shared=2), dict(lengths=[37, 20], parent=[0, 1], extra_held=2),
    dict(lengths=[37, 20], parent=[1, 0, 1], extra_held=2, room=30), dict(lengths=[37, 20], parent=[0, 0, 0, 1, 1], spare=2, room=17),
    dict(lengths=[37, 20], parent=[0, 0, 0, 1, 1], spare=0), dict(lengths=[200, 100], parent=[0, 0, 1], width_out=4), dict(lengths=[200, 100], parent=[1, 0], width_out=40),
    dict(lengths=[40, 41], parent=[0, 0, 1, 1], pool_kinds=("bf16", "bf16", "odd", "big")), dict(lengths=[40, 41], parent=[1, 1], pool_kinds=()),
    dict(lengths=[20 + 7 * (i % 30) for i in range(300)], parent=[(i * i) % 300 for i in range(400)], shared=1, spare=900, layers=1),
    dict(lengths=[5] * 3000, parent=[(i * 7) % 3000 // 2 for i in range(5000)], spare=6000, layers=1, pool_kinds=("odd",)),
    dict(lengths=[30000, 31000], parent=[0, 0, 0], shared=1800, spare=3000, layers=1, pool_kinds=("odd",)),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", range(len(FORKS)))
def test_fork_matches_the_oracle(case, in_place):
    kw = dict(FORKS[case])
    call = {k: kw.pop(k) for k in ("parent", "room", "width_out") if k in kw}
    Forest(seed=case, **kw).fork(in_place=in_place, **call)


def test_page_ids_outside_the_pools_are_passed_on():
    f = Forest([64, 40], spare=10)
    f.table[0][1], f.table[1][2] = -5, 10 ** 6
    f.refs = [max(x, 1) if x else 0 for x in f.refs]
    f.fork([0, 1, 1, 0])


def test_steps_of_a_beam_search_one_after_the_other():
    rng = np.random.default_rng(1)
    f = Forest([70] * 6, shared=4, spare=60)
    for step in range(12):
        f.fork(sorted(int(x) for x in rng.integers(0, len(f.held), int(rng.integers(1, 9)))), in_place=step % 2 == 0)
        f.length = [min(x + 1, 16 * h) for x, h in zip(f.length, f.held)]
        assert sum(r > 0 for r in f.refs) + len(f.free) == f.total


# ---------------------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_prompt_that_is_sampled_in_several_ways(dtype):
    """Prompt into 8-bit pages, three samples of it, tokens, a beam step, tokens: every attention against the dense history of its sequence."""
    t, hq, hkv, d, layers, pages, eps = TYPES[dtype], 8, 2, 128, 2, 64, 1e-6
    gen = torch.Generator(device="cuda").manual_seed(0)
    store = torch.full((layers, pages, hkv, 2, 16, d), 0x7f, dtype=torch.uint8, device="cuda").view(F8)
    scales = torch.full((layers, pages, hkv, 2), float("nan"), device="cuda")
    refs, free, count = torch.zeros(pages, dtype=torch.int32, device="cuda"), torch.arange(pages, dtype=torch.int32, device="cuda"), i32([pages])
    missing, ws = i32([0]), torch.zeros(pcb.OPS_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    gain = [1 + 0.2 * torch.randn(d, generator=gen, device="cuda") for _ in range(2)]
    angle = np.arange(256)[:, None] * 1e6 ** (-np.arange(d // 2) / (d // 2))
    rope = torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)).cuda()
    # an empty sequence that makes room for the prompt
    table, held, length = i32([[-1] * 12]), i32([0]), i32([0])
    history = [[np.zeros((2, 0, hkv, d)) for _ in range(layers)]]

    def fork(parent, room):
        nonlocal table, held, length, history
        m = len(parent)
        out = torch.zeros((m, 12), dtype=torch.int32, device="cuda"), torch.zeros(m, dtype=torch.int32, device="cuda"), torch.zeros(m, dtype=torch.int32, device="cuda")
        pcb.fork_pages(table, held, length, i32(parent), *out, refs, free, count, missing, pools=[store, scales], room=room, workspace=ws)
        table, held, length = out
        history = [[x.copy() for x in history[p]] for p in parent]
        assert missing.item() == 0

    def step(new):
        """`new` rows of every sequence through every layer: norms, rotation, store, attention."""
        nonlocal length
        n = len(history)
        row_start = i32([new * b for b in range(n + 1)])
        for layer in range(layers):
            x = torch.randn((n * new, hq + 2 * hkv, d), generator=gen, device="cuda").to(t)
            q = torch.empty((n * new, hq, d), dtype=t, device="cuda")
            pcb.append_rows(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], q, ctx_len=length, row_start=row_start, max_len=192, pages=store[layer],
                            scales=scales[layer], page_table=table, q_gain=gain[0], k_gain=gain[1], eps=eps, rope=rope)
            out, lse = torch.empty_like(q), torch.empty((n * new, hq), device="cuda")
            rows = min(new, 64)
            first = length + (new - rows)                    # the attention operator takes up to 256 rows of a sequence: the last ones here
            pcb.tree_attention_8bit(q.view(n, new, hq, d)[:, -rows:].reshape(-1, hq, d), store[layer], scales[layer], out[:n * rows], lse[:n * rows],
                                    ctx_len=first, row_start=i32([rows * b for b in range(n + 1)]), page_table=table, max_nodes=rows, max_len=192, workspace=ws)
            pcb.ops_status(ws)
            for b in range(n):
                c = int(length[b])
                tab = f64(rope)[c:c + new]
                xb = f64(x[b * new:(b + 1) * new])
                k = P.norm_rotate(xb[:, hq:hq + hkv], f64(gain[1]), eps, tab)
                history[b][layer] = np.concatenate([history[b][layer], np.stack([k, xb[:, hq + hkv:]])], 1)
                kv = history[b][layer]
                # what the pages hold is the history, rounded at most twice (a page's scale may have grown once over half its range) to 4 bits
                ids = table[b, :-(-(c + new) // 16)].long()
                have = P.VALUES[raw(store[layer][ids])] * f64(scales[layer][ids])[..., None, None]
                have = have.transpose(2, 0, 3, 1, 4).reshape(2, -1, hkv, d)[:, :c + new]
                step_size = f64(scales[layer][ids]).max() * 2.0 ** -9
                assert (np.abs(have - kv) <= np.abs(kv) * 2.0 ** -4 * 1.01 + step_size).all()
                want, _, mean_abs = ops.tree_attention(f64(q.view(n, new, hq, d)[b, -rows:]), have[0], have[1], c + new - rows, None, d ** -0.5)
                e = torch.finfo(t).eps / 2
                assert (np.abs(f64(out[b * rows:(b + 1) * rows]) - want) <= (e + 2.0 ** -12) * mean_abs + e * np.abs(want) + 2.0 ** -16 * np.abs(have).max()).all()
        length += new

    fork([0], 100)
    step(100)
    fork([0, 0, 0], 1)
    for _ in range(5):
        step(1)
        fork(list(range(len(history))), 1)
    fork([2, 0, 2, 2], 16)
    assert int((refs > 0).sum()) + count.item() == pages
    step(9)
    fork([3], 1)
    step(1)
    fork([], 0)
    assert count.item() == pages and int(refs.abs().sum()) == 0
    assert sorted(free.cpu().tolist()) == list(range(pages))
