"""Cases, plain forms and exact values of the operators that write, read and share the pages of a decoding batch's cache.

  append_rows          new rows of a batch on their way into the cache: RMS norms of the queries and keys head by head, the position
                       rotation, K and V stored in 16-bit pools or in 8-bit pages
  tree_attention_8bit  attention of new tokens (one a prompt, a chain, a drafted tree) over 8-bit pages
  fork_pages           the sequences of a batch continued by others (samples of one prompt, beams): page tables, counters, the
                       free list, and copies of the pages that two of them would write

An 8-bit page holds 16 slots: [kv_heads][K, V][16][head_dim] values of 4 exponent and 3 mantissa bits, and a scale (fp32) per KV head for K
and for V, by which they are multiplied.  append_rows takes the smallest power of two, within 2^-32 .. 2^32, with which
the largest value of the page's new rows is at most 448, or the page's present one where slots were in use and it is larger.
"""
import math

import torch

own = False

PAGE = 16
WORKSPACE_BYTES = 24 << 20
EPS = 1e-6
F8 = torch.float8_e4m3fn


# ------------------------------------------------------------------------------------------------------------ cases
def _append(name, **kw):
    c = {"name": name, "op": "append", "n_seqs": 1, "ctx": 0, "new": 1, "ragged": False, "q_heads": 16, "kv_heads": 8, "head_dim": 128,
         "dtype": "bf16", "cache": "8bit", "norm": True, "rope": True}
    c.update(kw)
    return c


def _attention(name, **kw):
    c = {"name": name, "op": "attention", "n_seqs": 1, "ctx": 2048, "ragged": False, "nodes": 1, "tree": "chain", "q_heads": 16,
         "kv_heads": 8, "head_dim": 128, "dtype": "bf16"}
    c.update(kw)
    return c


def _fork(name, **kw):
    c = {"name": name, "op": "fork", "n_seqs": 1, "ctx": 2112, "children": 4, "layers": 28, "kv_heads": 8, "head_dim": 128, "cache": "8bit",
         "room": 1, "shared": 0.75, "spread": 0.5}
    c.update(kw)
    return c


def listed():
    return [
        # one prompt's next token behind 2112 slots, into 16-bit pages: the smallest call, where latency counts
        _append("append_one_2112", ctx=2112, cache="pages"),
        # 64 ragged prompts, one token each, into 8-bit pages that are in part filled: the batched decode step
        _append("append_64x1_8bit", n_seqs=64, ctx=2500, ragged=True),
        # eight new prompts of ragged lengths, into 8-bit pages
        _append("append_8x2500_8bit", n_seqs=8, new=2500, ragged=True, dtype="f16"),
        # the 33024-token prompt, into a contiguous 16-bit context
        _append("append_33024", new=33024, cache="slots", dtype="f16"),
        # one prompt of 512 cached tokens, one new token
        _attention("decode8_one_512", ctx=511),
        # 64 ragged prompts around 2.5k tokens, one token each: the batched decode step
        _attention("decode8_64x2500", n_seqs=64, ctx=2500, ragged=True),
        # the same batch verifying ragged drafted trees of up to 26 nodes
        _attention("tree26_8bit_64x2500", n_seqs=64, ctx=2500, ragged=True, nodes=26, tree="tree"),
        # two 33024-token prompts, chains of 7 drafted tokens, four query heads a KV head
        _attention("chain7_8bit_2x33024", n_seqs=2, ctx=33024, nodes=7, q_heads=32, dtype="f16"),
        # four samples of one prompt of 2117 tokens, 28 layers of 8-bit pages
        _fork("fork_one_to_4", ctx=2117),
        # 16 beams of a 2112-token prompt, 28 layers of 8-bit pages: the usual step, some of them go on twice
        _fork("beams_16_8bit", n_seqs=16, children=16, spread=1.0),
        # 64 beams that go on from a quarter of them, 28 layers of 16-bit K and V pages
        _fork("beams_64_pages", n_seqs=64, children=64, cache="pages", spread=0.25),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(("append", "append", "append", "attention", "attention", "attention", "attention", "fork", "fork"))
    kv_heads = rng.choice((1, 2, 4, 8))
    more = {"kv_heads": kv_heads, "head_dim": rng.choice((64, 128, 128))}
    if op == "fork":
        n = _log_int(rng, 1, 64)
        c = _fork("", n_seqs=n, children=rng.choice((n, _log_int(rng, 1, 64))), ctx=_log_int(rng, 1, 4000), layers=_log_int(rng, 1, 28),
                  cache=rng.choice(("8bit", "pages")), room=rng.choice((0, 1, 1, 17)), shared=rng.random(), spread=rng.random(), **more)
        # pools of at most a gigabyte or so
        while n * c["ctx"] * c["layers"] * kv_heads * c["head_dim"] > 1.2e8 * 2:
            c["layers"], c["ctx"] = max(1, c["layers"] // 2), max(1, c["ctx"] * 2 // 3)
    else:
        more.update(q_heads=kv_heads * rng.choice((1, 2, 2, 3, 4, 8)), dtype=rng.choice(("f16", "bf16")), ragged=rng.random() < 0.5,
                    n_seqs=_log_int(rng, 1, 64))
        if op == "append":
            c = _append("", cache=rng.choice(("8bit", "8bit", "pages", "slots")), norm=rng.random() < 0.7, rope=rng.random() < 0.8, **more)
            c["new"] = rng.choice((1, _log_int(rng, 1, 20000 // c["n_seqs"])))
            c["ctx"] = rng.choice((0, _log_int(rng, 1, max(33024 // c["n_seqs"] - c["new"], 1))))
            while c["q_heads"] > 32:
                c["q_heads"] //= 2
        else:
            c = _attention("", tree=rng.choice(("tree", "chain")), nodes=rng.choice((1, 1, _log_int(rng, 2, 64))), **more)
            c["ctx"] = _log_int(rng, 1, min(33024, 100000 // c["n_seqs"]))
            while c["n_seqs"] * c["ctx"] * c["nodes"] * c["q_heads"] > 64 * 2500 * 26 * 16:
                c["nodes"] = max(1, c["nodes"] // 2)
    del c["name"]
    return c


def _spread(n, ragged, what, low, high):
    """`what` a prompt, or low .. high times it."""
    golden = 0.6180339887498949
    return [int(what * (low + (high - low) * ((b * golden) % 1.0))) if ragged else what for b in range(n)]


def _lengths(case):
    """Slots in use and new rows of every prompt: from the case alone."""
    n, ragged = case["n_seqs"], case["ragged"]
    new = case["new"] if case["op"] == "append" else case["nodes"]
    return _spread(n, ragged, case["ctx"], 0.4, 1.6), [max(1, x) for x in _spread(n, ragged, new, 0.25, 1.0)[::-1]]


# ------------------------------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.float16 if case.get("dtype") == "f16" else torch.bfloat16


def _tables(pages, gen, spare=3):
    """A page table [prompts, most pages] of shuffled page ids, and how many pages the pools have."""
    total = sum(pages) + spare
    order = torch.randperm(total, generator=gen, dtype=torch.int32)
    t = torch.zeros((len(pages), max(max(pages), 1)), dtype=torch.int32)
    at = 0
    for b, p in enumerate(pages):
        t[b, :p] = order[at:at + p]
        at += p
    return t, order, total


def _tree_mask(nodes, gen):
    """Rows of 64-bit words: node i sees itself and its ancestors in a random tree."""
    words = -(-max(nodes) // 64)
    rows = []
    for n in nodes:
        r = torch.rand(n, generator=gen).tolist()
        seen = []
        for i in range(n):
            parent = int(r[i] * (i + 1)) - 1          # -1: a child of the context's last token
            seen.append((seen[parent] if parent >= 0 else 0) | (1 << i))
            w = [(seen[i] >> (64 * k)) & (2 ** 64 - 1) for k in range(words)]
            rows.append([x - 2 ** 64 if x >= 2 ** 63 else x for x in w])
    return torch.tensor(rows, dtype=torch.int64).cuda()


def _random_pages(total, case, dev):
    """8-bit pages of normal values, the heads' sizes apart by up to a factor of four, and their scales."""
    shape = (total, case["kv_heads"], 2, PAGE, case["head_dim"])
    scales = torch.exp2(torch.randint(-9, -6, shape[:3], generator=dev, device="cuda").float())
    x = torch.randn(shape, generator=dev, device="cuda").mul_(112.0).clamp_(-448, 448)
    return x.to(F8), scales


def prepare(case, seed):
    gen = torch.Generator().manual_seed(seed)
    dev = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "fork":
        return _prepare_fork(case, gen, dev)
    ctx, new = _lengths(case)
    hkv, hq, d, n, t = case["kv_heads"], case["q_heads"], case["head_dim"], case["n_seqs"], _dtype(case)
    lens = [a + b for a, b in zip(ctx, new)]
    rows = sum(new)
    s = {"case": case, "max_len": max(lens), "ctx_len": torch.tensor(ctx, dtype=torch.int32).cuda(),
         "row_start": torch.tensor([sum(new[:b]) for b in range(n + 1)], dtype=torch.int32).cuda(), "max_new": max(new)}
    paged = case["op"] == "attention" or case["cache"] != "slots"
    if paged:
        table, _, total = _tables([-(-x // PAGE) for x in lens], gen)
        s["page_table"] = table.cuda()
    else:
        s["ctx_start"] = torch.tensor([5 + sum(lens[:b]) for b in range(n)], dtype=torch.int32).cuda()
        total = -(-(sum(lens) + 5) // PAGE)
    if case["op"] == "attention" or case["cache"] == "8bit":
        s["pages"], s["scales"] = _random_pages(total, case, dev)
    else:
        s["k_pool"] = torch.randn((total * PAGE, hkv, d), generator=dev, device="cuda").to(t)
        s["v_pool"] = torch.randn((total * PAGE, hkv, d), generator=dev, device="cuda").to(t)
    if case["op"] == "append":
        # the projection's output, queries, keys and values of a row side by side; keys of a few channels are larger
        qkv = torch.randn((rows, hq + 2 * hkv, d), generator=dev, device="cuda")
        qkv[:, hq:hq + hkv, ::17] *= 4
        s["qkv"] = qkv.to(t)
        s["q_out"] = torch.zeros((rows, hq, d), dtype=t, device="cuda")
        s["q_gain"] = (1 + 0.3 * torch.randn(d, generator=dev, device="cuda")) if case["norm"] else None
        s["k_gain"] = (1 + 0.3 * torch.randn(d, generator=dev, device="cuda")) if case["norm"] else None
        s["rope"] = None
        if case["rope"]:
            angle = torch.arange(s["max_len"], dtype=torch.float64, device="cuda")[:, None] * torch.exp2(
                -math.log2(1e6) / (d // 2) * torch.arange(d // 2, dtype=torch.float64, device="cuda"))
            s["rope"] = torch.stack((angle.cos(), angle.sin()), -1).float()
        return s
    s["mask"] = _tree_mask(new, gen) if case["tree"] == "tree" else None
    s["scale"] = d ** -0.5
    s["q"] = (2.0 * torch.randn((rows, hq, d), generator=dev, device="cuda")).to(t)
    s["out"] = torch.zeros((rows, hq, d), dtype=t, device="cuda")
    s["lse"] = torch.zeros((rows, hq), dtype=torch.float32, device="cuda")
    s["workspace"] = torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    return s


def _fork_sizes(case):
    """Length and held pages of every sequence, and how many leading pages all of them share: from the case alone."""
    n, ctx = case["n_seqs"], case["ctx"]
    lens = [max(1, ctx - (b * 7) % 16 if ctx > 16 else ctx) for b in range(n)]
    held = [-(-x // PAGE) for x in lens]
    return lens, held, min(int(case["shared"] * ctx) // PAGE, min(lens) // PAGE) if n > 1 else 0


def _parents(case):
    """The sequence that each child continues.  spread 1: the children of a beam search's usual step, two in three sequences go on."""
    n, m = case["n_seqs"], case["children"]
    golden = 0.6180339887498949
    return [int(n * case["spread"] * ((i * golden) % 1.0) ** 1.5) % n for i in range(m)]


def _prepare_fork(case, gen, dev):
    lens, held, shared = _fork_sizes(case)
    n, m, hkv, d, layers = case["n_seqs"], case["children"], case["kv_heads"], case["head_dim"], case["layers"]
    private, order, total = _tables([h - shared for h in held], gen, spare=shared + m * (2 + case["room"] // PAGE) + 5)
    width = max(held) + 2 + case["room"] // PAGE
    table = torch.full((n, width), -1, dtype=torch.int32)
    used = sum(held) - shared * n
    table[:, :shared] = order[used:used + shared]
    for b in range(n):
        table[b, shared:held[b]] = private[b, :held[b] - shared]
    refs = torch.zeros(total, dtype=torch.int32)
    refs[order[:used].long()] = 1
    refs[order[used:used + shared].long()] = n
    free = torch.full((total,), -1, dtype=torch.int32)
    spare = order[used + shared:]
    free[:len(spare)] = spare
    s = {"case": case, "page_table": table.cuda(), "held": torch.tensor(held, dtype=torch.int32).cuda(),
         "length": torch.tensor(lens, dtype=torch.int32).cuda(), "parent": torch.tensor(_parents(case), dtype=torch.int32).cuda(),
         "refs": refs.cuda(), "free_list": free.cuda(), "free_count": torch.tensor([len(spare)], dtype=torch.int32).cuda(),
         "workspace": torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")}
    for name in ("refs", "free_list", "free_count"):
        s[name + "_out"] = torch.zeros_like(s[name])
    s["table_out"] = torch.zeros((m, width), dtype=torch.int32, device="cuda")
    s["held_out"] = torch.zeros(m, dtype=torch.int32, device="cuda")
    s["length_out"] = torch.zeros(m, dtype=torch.int32, device="cuda")
    s["missing"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if case["cache"] == "8bit":
        page = torch.randint(0, 0x78, (layers, total, hkv, 2, PAGE, d), generator=dev, device="cuda", dtype=torch.uint8)
        s["pools"] = [page.view(F8), torch.rand((layers, total, hkv, 2), generator=dev, device="cuda")]
    else:
        s["pools"] = [torch.randint(0, 0x3c00, (layers, total, PAGE, hkv, d), generator=dev, device="cuda", dtype=torch.int16).view(torch.bfloat16)
                      for _ in range(2)]
    return s


# ------------------------------------------------------------------------------------------------------------ plain forms
def _slots(s, width):
    """Pool rows [n_seqs, width] of slots 0 .. width - 1 (those past a prompt's length are not used)."""
    t = torch.arange(width, device="cuda")
    if "page_table" in s:
        return s["page_table"].long()[:, (t // PAGE).clamp(max=s["page_table"].shape[1] - 1)] * PAGE + t % PAGE
    return s["ctx_start"].long()[:, None] + t


def _owner(s, rows):
    """Prompt and slot of every row."""
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(s["row_start"].long(), r, right=True) - 1
    return b, s["ctx_len"].long()[b] + r - s["row_start"].long()[b]


def _norm_rotate(x, gain, table):
    """x [rows, heads, d], gain [d] or None, table [rows, d / 2, (cos, sin)] or None."""
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.to(x.dtype)
    if table is not None:
        c, sn = table.to(x.dtype)[:, None, :, 0], table.to(x.dtype)[:, None, :, 1]
        a, b = x.chunk(2, -1)
        x = torch.cat((a * c - b * sn, b * c + a * sn), -1)
    return x


def _append_plain(s):
    case = s["case"]
    hq, hkv, t = case["q_heads"], case["kv_heads"], _dtype(case)
    rows = s["qkv"].shape[0]
    b, slot = _owner(s, rows)
    table = s["rope"][slot] if s["rope"] is not None else None
    s["q_out"].copy_(_norm_rotate(s["qkv"][:, :hq].float(), s["q_gain"], table))
    eight = case["cache"] == "8bit"
    wide = torch.float64 if eight else torch.float32          # 64 bits where values next to a border of 8 bits count
    k = _norm_rotate(s["qkv"][:, hq:hq + hkv].to(wide), s["k_gain"], table)
    v = s["qkv"][:, hq + hkv:].to(wide)
    if not eight:
        at = _slots(s, s["max_len"])[b, slot]
        s["k_pool"][at] = k.to(t)
        s["v_pool"][at] = v.to(t)
        return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}
    # the touched pages of every prompt, [prompts, most pages of one]
    x = torch.stack((k, v), 2)                                                        # [rows, hkv, 2, d]
    ctx, first = s["ctx_len"].long(), s["row_start"].long()
    n_new = first[1:] - first[:-1]
    most = s["max_new"] // PAGE + 2
    page = ctx[:, None] // PAGE + torch.arange(most, device="cuda")
    slots = page[:, :, None] * PAGE + torch.arange(PAGE, device="cuda")                # [n, most, 16]
    is_new = (slots >= ctx[:, None, None]) & (slots < (ctx + n_new)[:, None, None])
    is_old = slots < ctx[:, None, None]
    touched = is_new.any(-1) & (n_new > 0)[:, None]
    row = (first[:-1, None, None] + slots - ctx[:, None, None])[touched].clamp(0, rows - 1)
    is_new, is_old = is_new[touched], is_old[touched]                                  # [p, 16]
    pid = torch.gather(s["page_table"].long(), 1, page.clamp(max=s["page_table"].shape[1] - 1))[touched]
    new = x[row].permute(0, 2, 3, 1, 4)                                                # [p, hkv, 2, 16, d]
    fresh = is_new[:, None, None, :, None]
    amax = torch.where(fresh, new.abs(), torch.zeros((), dtype=wide, device="cuda")).amax((-1, -2))
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 9 + (m > 0.875).to(e.dtype), torch.full_like(e, -32)).clamp(-32, 32)
    scale = torch.ldexp(torch.ones_like(amax), e)
    before = s["scales"][pid].to(wide)
    scale = torch.where(is_old.any(-1)[:, None, None], torch.maximum(scale, before), scale)
    held = s["pages"][pid]
    again = (held.to(wide) * (before / scale)[..., None, None]).clamp(-448, 448).float().to(F8)
    put = (new / scale[..., None, None]).clamp(-448, 448).float().to(F8)
    raw = torch.where(fresh, put.view(torch.uint8), torch.where(is_old[:, None, None, :, None], again.view(torch.uint8), held.view(torch.uint8)))
    s["pages"].view(torch.uint8)[pid] = raw
    s["scales"][pid] = scale.float()
    return {"q": s["q_out"], "pages": s["pages"], "scales": s["scales"]}


def _attention_plain(s):
    n, (hq, d) = s["ctx_len"].numel(), s["q"].shape[1:]
    hkv = s["pages"].shape[1]
    m, t = s["max_new"], s["max_len"]
    ctx, first = s["ctx_len"].long(), s["row_start"].long()
    count = first[1:] - first[:-1]
    node = torch.arange(m, device="cuda")
    slot = torch.arange(t, device="cuda")
    real = node < count[:, None]                                                      # [n, m]
    row = torch.where(real, first[:-1, None] + node, first[:-1, None])
    j = slot - ctx[:, None]                                                           # [n, t]: the slot's node, or negative
    if s["mask"] is not None:
        jc = j.clamp(0, m - 1)
        words = s["mask"][row]                                                        # [n, m, words]
        word = torch.gather(words, 2, (jc >> 6)[:, None, :].expand(n, m, t))
        node_seen = ((word >> (jc & 63)[:, None, :]) & 1) != 0
    else:
        node_seen = j[:, None, :] <= node[None, :, None]
    seen = (j < 0)[:, None, :] | ((j < count[:, None])[:, None, :] & node_seen & (j >= 0)[:, None, :])
    seen = seen & real[:, :, None]
    pid = s["page_table"].long()
    kv = s["pages"][pid].float() * s["scales"][pid][..., None, None]                   # [n, pages, hkv, 2, 16, d]
    kv = kv.permute(3, 0, 2, 1, 4, 5).reshape(2, n, hkv, -1, d)[:, :, :, :t]
    g = hq // hkv
    qf = s["q"][row].float().view(n, m, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, d)
    x = torch.matmul(qf, kv[0].transpose(-1, -2)).view(n, hkv, m, g, t) * s["scale"]
    x = x.masked_fill(~seen[:, None, :, None, :], -math.inf)
    any_seen = seen.any(-1)[:, None, :, None, None]
    top = torch.where(any_seen, x.amax(-1, keepdim=True), torch.zeros((), device="cuda"))
    x = torch.exp(x - top)
    total = x.sum(-1)                                                                 # [n, hkv, m, g]
    inside = slot < (ctx + count)[:, None]
    vf = torch.where(inside[:, None, :, None], kv[1], torch.zeros((), device="cuda"))
    o = torch.matmul(x.view(n, hkv, m * g, t), vf).view(n, hkv, m, g, d)
    o = torch.where(any_seen, o / total[..., None], torch.zeros((), device="cuda"))
    lse = torch.log(total) + top[..., 0]
    s["out"][row[real]] = o.permute(0, 2, 1, 3, 4).reshape(n, m, hq, d)[real].to(s["q"].dtype)
    s["lse"][row[real]] = lse.permute(0, 2, 1, 3).reshape(n, m, hq)[real]
    return {"out": s["out"], "lse": s["lse"]}


def _fork_plain(s):
    room = s["case"]["room"]
    n, width = s["page_table"].shape
    m, wide = s["table_out"].shape
    total = s["refs"].numel()
    held = s["held"].long().clamp(0, width)
    length = torch.minimum(s["length"].long().clamp(min=0), held * PAGE)
    ok = (s["parent"] >= 0) & (s["parent"] < n)
    p = s["parent"].long().clamp(0, n - 1)
    child = torch.arange(m, device="cuda")
    first = torch.full((n,), m, device="cuda").scatter_reduce(0, p, torch.where(ok, child, m), "amin")
    heir = ok & (first[p] == child)                    # the first child goes on with the sequence's own last page
    full, part = length[p] // PAGE, length[p] % PAGE > 0
    have = torch.where(ok, torch.where(heir, held[p], full), 0).clamp(max=wide)
    want = torch.where(ok, (length[p] + room + PAGE - 1) // PAGE, 0).clamp(max=wide)
    fresh = (want - have).clamp(min=0)
    start = fresh.cumsum(0) - fresh
    count = s["free_count"].long()
    got = torch.minimum((count - start).clamp(min=0), fresh)
    j = torch.arange(wide, device="cuda")
    k = count - 1 - (start[:, None] + j - have[:, None])                                # place in the free list
    new = j < (have + got)[:, None]
    kept = j < have[:, None]
    inherited = torch.nn.functional.pad(s["page_table"].long(), (0, max(wide - width, 0)), value=-1)[p][:, :wide]
    table = torch.where(kept, inherited, torch.where(new, s["free_list"].long()[k.clamp(0, total - 1)], -1))
    s["table_out"].copy_(table)
    s["held_out"].copy_(have + got)
    s["length_out"].copy_(torch.where(ok, torch.minimum(length[p], (have + got) * PAGE), 0))
    s["missing"].copy_((fresh - got).sum())
    # counters: a sequence's full pages are shared by its children; without a child all its pages lose one holder
    children = torch.zeros(n, dtype=torch.long, device="cuda").scatter_add(0, p, ok.long())
    i = torch.arange(width, device="cuda")
    of_full = i < (length // PAGE)[:, None]
    delta = torch.where(children[:, None] == 0, -1, torch.where(of_full, children[:, None] - 1, 0))
    delta = torch.where(i < held[:, None], delta, 0)
    refs = s["refs"].long().scatter_add(0, s["page_table"].long().clamp(0, total - 1).reshape(-1), delta.reshape(-1))
    freed = (s["refs"] > 0) & (refs == 0)
    taken = table[new & ~kept]
    refs[taken] = 1
    s["refs_out"].copy_(refs)
    base = count - taken.numel()
    freed_ids = torch.nonzero(freed)[:, 0]                                             # ascending
    s["free_list_out"].copy_(s["free_list"])
    s["free_list_out"][base + torch.arange(freed_ids.numel(), device="cuda")] = freed_ids.to(torch.int32)
    s["free_count_out"].copy_(base + freed_ids.numel())
    copied = ok & ~heir & part & (got > 0)
    src, dst = inherited.gather(1, full[:, None])[copied, 0], table.gather(1, full[:, None].clamp(max=wide - 1))[copied, 0]
    both = [x.view(torch.uint8) if x.dtype == F8 else x for x in s["pools"]]
    both[0][:, dst] = both[0][:, src]
    both[1][:, dst] = both[1][:, src]
    return _fork_outputs(s)


def _fork_outputs(s):
    return {"table": s["table_out"], "held": s["held_out"], "length": s["length_out"], "refs": s["refs_out"], "free_list": s["free_list_out"],
            "free_count": s["free_count_out"], "missing": s["missing"], "pool0": s["pools"][0].view(torch.int16),
            "pool1": s["pools"][1].view(torch.int32)}


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2601_11553_b200 import percache as pc
        if op == "append":
            hq, hkv = s["case"]["q_heads"], s["case"]["kv_heads"]
            qkv = s["qkv"]
            pc.append_rows(qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], s["q_out"], ctx_len=s["ctx_len"], row_start=s["row_start"],
                           max_len=s["max_len"], k_pool=s.get("k_pool"), v_pool=s.get("v_pool"), pages=s.get("pages"), scales=s.get("scales"),
                           page_table=s.get("page_table"), ctx_start=s.get("ctx_start"), q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS,
                           rope=s["rope"])
            if "pages" in s:
                return {"q": s["q_out"], "pages": s["pages"], "scales": s["scales"]}
            return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}
        if op == "attention":
            pc.tree_attention_8bit(s["q"], s["pages"], s["scales"], s["out"], s["lse"], ctx_len=s["ctx_len"], row_start=s["row_start"],
                                   page_table=s["page_table"], mask=s["mask"], max_nodes=s["max_new"], max_len=s["max_len"],
                                   scale=s["scale"], workspace=s["workspace"])
            return {"out": s["out"], "lse": s["lse"]}
        pc.fork_pages(s["page_table"], s["held"], s["length"], s["parent"], s["table_out"], s["held_out"], s["length_out"], s["refs"],
                      s["free_list"], s["free_count"], s["missing"], pools=s["pools"], room=s["case"]["room"], refs_out=s["refs_out"],
                      free_list_out=s["free_list_out"], free_count_out=s["free_count_out"], workspace=s["workspace"])
        return _fork_outputs(s)
    if op == "append":
        return _append_plain(s)
    if op == "attention":
        return _attention_plain(s)
    return _fork_plain(s)


# ------------------------------------------------------------------------------------------------------------ least work
def work(case):
    hkv, d = case["kv_heads"], case["head_dim"]
    if case["op"] == "fork":
        lens, held, _ = _fork_sizes(case)
        seen, copies = set(), 0
        for p in _parents(case):
            copies += p in seen and lens[p] % PAGE > 0
            seen.add(p)
        page = case["layers"] * (hkv * (2 * PAGE * d + 8) if case["cache"] == "8bit" else 4 * PAGE * hkv * d)
        children = [held[p] for p in _parents(case)]
        return {"bytes": 2 * copies * page + 4 * (sum(held) + sum(children)) + 16 * case["children"], "flops": 0}
    ctx, new = _lengths(case)
    hq, n, rows = case["q_heads"], case["n_seqs"], sum(new)
    lens = [a + b for a, b in zip(ctx, new)]
    if case["op"] == "append":
        pages = sum((a + b + PAGE - 1) // PAGE - a // PAGE for a, b in zip(ctx, new))
        stored = 2 * hkv * (rows * d + pages * 4) if case["cache"] == "8bit" else 4 * hkv * rows * d
        table = min(max(lens), rows) * d * 4 if case["rope"] else 0
        return {"bytes": rows * d * (4 * hq + 4 * hkv) + stored + table + 4 * pages + 8 * n,
                "flops": rows * d * (hq + hkv) * (4 * case["norm"] + 3 * case["rope"])}
    pages = sum(-(-t // PAGE) for t in lens)
    return {"bytes": sum(lens) * hkv * d * 2 + pages * (hkv * 8 + 4) + rows * hq * (4 * d + 4) + 8 * n,
            "flops": 4 * d * hq * sum(m * (t + 1) for m, t in zip(new, ctx))}


# ------------------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """Prompt by prompt, straight from the definitions.  8-bit values are given before their rounding."""
    if case["op"] == "fork":
        return None                    # whole numbers, and values that are only moved
    s = prepare(case, seed)
    ctx, new = _lengths(case)
    hkv, hq, d = case["kv_heads"], case["q_heads"], case["head_dim"]
    g = hq // hkv
    table = s["page_table"].cpu().tolist() if "page_table" in s else None
    r0 = 0
    if case["op"] == "append":
        def rotated(x, gain, b):
            if gain is not None:
                x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / d + EPS) * gain.double()
            if s["rope"] is not None:
                z = torch.complex(x[..., :d // 2], x[..., d // 2:]) * torch.view_as_complex(s["rope"][ctx[b]:ctx[b] + new[b]].double())[:, None]
                x = torch.cat((z.real, z.imag), -1)
            return x

        q = torch.zeros((sum(new), hq, d), dtype=torch.float64, device="cuda")
        eight = case["cache"] == "8bit"
        if eight:
            pages, scales = s["pages"].to(torch.float64), s["scales"].double()
        else:
            pools = [s["k_pool"].double(), s["v_pool"].double()]
        for b in range(case["n_seqs"]):
            x = s["qkv"][r0:r0 + new[b]].double()
            q[r0:r0 + new[b]] = rotated(x[:, :hq], s["q_gain"], b)
            kv = (rotated(x[:, hq:hq + hkv], s["k_gain"], b), x[:, hq + hkv:])
            if not eight:
                slots = torch.arange(ctx[b], ctx[b] + new[b], device="cuda")
                at = s["page_table"][b].long()[slots // PAGE] * PAGE + slots % PAGE if table else slots + int(s["ctx_start"][b])
                pools[0][at], pools[1][at] = kv
            else:
                for j in range(ctx[b] // PAGE, -(-(ctx[b] + new[b]) // PAGE)):
                    lo, hi = max(j * PAGE, ctx[b]), min(j * PAGE + PAGE, ctx[b] + new[b])
                    page = table[b][j]
                    for w in (0, 1):
                        rows = kv[w][lo - ctx[b]:hi - ctx[b]].transpose(0, 1)           # [hkv, slots, d]
                        e = torch.ceil(torch.log2(rows.abs().amax((1, 2)) / 448)).clamp(-32, 32)
                        scale = 2.0 ** e
                        if lo > j * PAGE:
                            before = scales[page, :, w].clone()
                            scale = torch.maximum(scale, before)
                            pages[page, :, w, :lo - j * PAGE] *= (before / scale)[:, None, None]
                        pages[page, :, w, lo - j * PAGE:hi - j * PAGE] = rows / scale[:, None, None]
                        scales[page, :, w] = scale
            r0 += new[b]
        return {"q": q, "pages": pages, "scales": scales} if eight else {"q": q, "k": pools[0], "v": pools[1]}
    out = torch.zeros((sum(new), hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((sum(new), hq), dtype=torch.float64, device="cuda")
    for b in range(case["n_seqs"]):
        c, m = ctx[b], new[b]
        t = c + m
        hidden = torch.zeros((m, t), dtype=torch.bool)
        if s["mask"] is None:
            hidden[:, c:] = torch.ones((m, m)).triu(1).bool()
        else:
            words = s["mask"][r0:r0 + m].cpu().tolist()
            for i in range(m):
                for j in range(m):
                    hidden[i, c + j] = not (words[i][j // 64] >> (j % 64)) & 1
        hidden = hidden.cuda()
        pid = s["page_table"][b, :-(-t // PAGE)].long()
        for h in range(hkv):
            k, v = ((s["pages"][pid, h, w].double() * s["scales"][pid, h, w].double()[:, None, None]).reshape(-1, d)[:t] for w in (0, 1))
            for q in range(h * g, (h + 1) * g):
                x = (s["q"][r0:r0 + m, q].double() @ k.T) * s["scale"]
                x[hidden] = -math.inf
                lse[r0:r0 + m, q] = torch.logsumexp(x, -1)
                out[r0:r0 + m, q] = torch.softmax(x, -1) @ v
        r0 += m
    return {"out": out, "lse": lse}
