"""Cases, plain forms and exact values of the operators that work on a decoding batch's cache.

  tree_attention     attention of drafted tokens (a tree, a chain, or one token a prompt) over the prompt's cached
                     context and the drafted tokens that each of them may see
  attention_weights  the softmax weights of the accepted rows, summed into one running value per KV head and slot
  select_slots       the slots to keep under a budget: the first, the most recent, and the heaviest of the rest
  compact_slots      the kept slots' K, V and running weights moved together, head by head

A batch is ragged: prompt b has ctx_len[b] cached slots and row_start[b + 1] - row_start[b] drafted tokens (nodes),
whose K and V sit in the slots right behind.  A slot of prompt b is a row of the K and V pools: through a table of
16-slot pages, or contiguous from ctx_start[b] on.  Node i sees every cached slot and the nodes j whose bit is set in
its row of `mask` (64 nodes a word); without a mask, the nodes up to itself.
"""
import math

import torch

own = False

PAGE = 16
WORKSPACE_BYTES = 24 << 20


# ------------------------------------------------------------------------------------------------------------ cases
def _case(name, op, **kw):
    c = {"name": name, "op": op, "n_seqs": 1, "ctx": 2048, "ragged": False, "nodes": 1, "tree": "chain", "q_heads": 16,
         "kv_heads": 8, "head_dim": 128, "dtype": "f16", "paged": False}
    c.update(kw)
    return c


def listed():
    return [
        # one prompt of 512 cached tokens, one new token: the shortest decode step, where only latency counts
        _case("decode_one_512", "tree", ctx=512, nodes=1),
        # the 2112-token prompt with a drafted tree of 26 nodes, K and V in pages
        _case("tree26_2112_paged", "tree", ctx=2112, nodes=26, tree="tree", dtype="bf16", paged=True),
        # 64 ragged prompts around 2.5k tokens, one token each: the batched decode step
        _case("decode_64x2500", "tree", n_seqs=64, ctx=2500, ragged=True, nodes=1),
        # the same batch verifying ragged trees of up to 48 nodes, K and V in pages
        _case("tree48_64x2500_paged", "tree", n_seqs=64, ctx=2500, ragged=True, nodes=48, tree="tree", dtype="bf16", paged=True),
        # two 33024-token prompts with a chain of 7 drafted tokens, four query heads a KV head
        _case("chain7_2x33024", "tree", n_seqs=2, ctx=33024, nodes=7, q_heads=32, dtype="bf16"),
        # running weights of one token on the 2112-token prompt
        _case("weights_one_2112", "weights", ctx=2112, nodes=1),
        # the batched decode step's weights, K in pages
        _case("weights_64x2500_paged", "weights", n_seqs=64, ctx=2500, ragged=True, nodes=1, dtype="bf16", paged=True),
        # two long prompts, the accepted half of 33 drafted tokens
        _case("weights33_2x33024", "weights", n_seqs=2, ctx=33024, nodes=33, tree="tree", dtype="bf16", paged=True),
        # the 28 layers of the 2112-token prompt, cut to 1024 slots
        _case("select_28x2112", "select", n_seqs=28, ctx=2112, budget=1024, sink=4, recent=128),
        # the 28 layers of the 33024-token prompt, cut to 8192 slots
        _case("select_28x33024", "select", n_seqs=28, ctx=33024, budget=8192, sink=16, recent=1001),
        # one prompt's layer of 2112 slots, 1024 of them moved to other pages
        _case("compact_2112_paged", "compact", ctx=2112, budget=1024, sink=4, recent=128, dtype="bf16", paged=True),
        # seven layers of the 33024-token prompt, a quarter of the slots kept
        _case("compact_7x33024", "compact", n_seqs=7, ctx=33024, budget=8192, sink=16, recent=1001),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(("tree", "tree", "tree", "weights", "weights", "select", "compact"))
    kv_heads = rng.choice((1, 2, 4, 8))
    c = _case("", op, kv_heads=kv_heads, q_heads=kv_heads * rng.choice((1, 2, 2, 3, 4, 8)), head_dim=rng.choice((64, 128, 128)),
              dtype=rng.choice(("f16", "bf16")), paged=rng.random() < 0.5, tree=rng.choice(("tree", "chain")),
              nodes=rng.choice((1, 1, _log_int(rng, 2, 64))), ragged=rng.random() < 0.5, n_seqs=_log_int(rng, 1, 64))
    c["ctx"] = _log_int(rng, 1, min(33024, 100000 // c["n_seqs"]))
    if op in ("select", "compact"):
        c["budget"] = _log_int(rng, 1, c["ctx"])
        c["sink"] = rng.randint(0, c["budget"] // 4)
        c["recent"] = rng.randint(0, c["budget"] // 2)
    else:
        # the plain form lays every prompt out at the longest one's length, with all scores at once
        while c["n_seqs"] * c["ctx"] * c["nodes"] * c["q_heads"] > 64 * 2500 * 48 * 16:
            c["nodes"] = max(1, c["nodes"] // 2)
    del c["name"]
    return c


def _lengths(case):
    """ctx_len and node count of every prompt: from the case alone."""
    n = case["n_seqs"]
    if not case["ragged"]:
        return [case["ctx"]] * n, [case["nodes"]] * n
    golden = 0.6180339887498949
    ctx = [int(case["ctx"] * (0.4 + 1.2 * ((b * golden) % 1.0))) for b in range(n)]
    nodes = [max(1, int(round(case["nodes"] * (0.25 + 0.75 * ((b * golden + 0.5) % 1.0))))) for b in range(n)]
    return ctx, nodes


def _used(case, i):
    return i % 2 == 0          # attention_weights: the rows that count (the accepted ones)


# ------------------------------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.float16 if case["dtype"] == "f16" else torch.bfloat16


def _places(case, lens, gen, spare):
    """Rows of the pools for prompts of `lens` slots: {"page_table"} or {"ctx_start"}, and the pools' row count.  `spare`:
    the same again, elsewhere in the pools."""
    n = len(lens)
    if case["paged"]:
        pages = [-(-t // PAGE) for t in lens]
        width = max(max(pages), 1)
        total = sum(pages) * (2 if spare else 1) + 3
        order = torch.randperm(total, generator=gen, dtype=torch.int32)
        tables, at = [], 0
        for _ in range(2 if spare else 1):
            t = torch.zeros((n, width), dtype=torch.int32)
            for b in range(n):
                t[b, :pages[b]] = order[at:at + pages[b]]
                at += pages[b]
            tables.append(t)
        return {"page_table": tables[0].cuda(), "dst_page_table": tables[1].cuda() if spare else None}, total * PAGE
    starts, at = [], 5
    for _ in range(2 if spare else 1):
        s = []
        for t in lens:
            s.append(at)
            at += t
        starts.append(torch.tensor(s, dtype=torch.int32).cuda())
    return {"ctx_start": starts[0], "dst_start": starts[1] if spare else None}, at


def _tree_mask(case, nodes, gen):
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


def prepare(case, seed):
    gen = torch.Generator().manual_seed(seed)
    dev = torch.Generator(device="cuda").manual_seed(seed)
    ctx, nodes = _lengths(case)
    hkv, hq, d, n = case["kv_heads"], case["q_heads"], case["head_dim"], case["n_seqs"]
    s = {"case": case, "workspace": torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")}

    def weights(width):
        # running sums with decay after a few hundred steps: a few heavy slots, a long tail, slots that never got any, and
        # about eight steps' worth of softmax weight of two query heads in all
        w = torch.rand((n, hkv, width), generator=dev, device="cuda").pow(8) * (144.0 / width)
        w[torch.rand((n, hkv, width), generator=dev, device="cuda") < 0.2] = 0
        return w

    if case["op"] == "select":
        s["length"] = torch.tensor(ctx, dtype=torch.int32).cuda()
        s["max_len"] = max(max(ctx), 1)
        s["weights"] = weights(s["max_len"])
        s["keep"] = torch.empty((n, hkv, case["budget"]), dtype=torch.int32, device="cuda")
        s["count"] = torch.empty(n, dtype=torch.int32, device="cuda")
        return s

    drafted = case["op"] in ("tree", "weights")
    lens = [a + (b if drafted else 0) for a, b in zip(ctx, nodes)]
    places, rows = _places(case, lens, gen, case["op"] == "compact")
    s.update(places)
    s["max_len"] = max(max(lens), 1)
    s["k"] = torch.randn((rows, hkv, d), generator=dev, device="cuda").to(_dtype(case))
    s["v"] = torch.randn((rows, hkv, d), generator=dev, device="cuda").to(_dtype(case))
    if case["op"] == "compact":
        s["weights"] = weights(s["max_len"])
        s["weights_out"] = torch.zeros_like(s["weights"])
        length = torch.tensor(ctx, dtype=torch.int32).cuda()
        s["keep"], s["count"] = _select_plain(s["weights"], length, case["budget"], case["sink"], case["recent"])
        return s

    total = sum(nodes)
    s["ctx_len"] = torch.tensor(ctx, dtype=torch.int32).cuda()
    s["row_start"] = torch.tensor([sum(nodes[:b]) for b in range(n + 1)], dtype=torch.int32).cuda()
    s["max_nodes"] = max(nodes)
    s["mask"] = _tree_mask(case, nodes, gen) if case["tree"] == "tree" else None
    s["scale"] = d ** -0.5
    s["q"] = (2.0 * torch.randn((total, hq, d), generator=dev, device="cuda")).to(_dtype(case))
    if case["op"] == "tree":
        s["out"] = torch.zeros((total, hq, d), dtype=_dtype(case), device="cuda")
        s["lse"] = torch.zeros((total, hq), dtype=torch.float32, device="cuda")
    else:
        s["lse"] = _tree_plain(s)["lse"]
        s["use"] = torch.tensor([_used(case, i) for m in nodes for i in range(m)], dtype=torch.uint8).cuda()
        s["weights"] = weights(s["max_len"])
        s["weights_out"] = torch.zeros_like(s["weights"])
    return s


# ------------------------------------------------------------------------------------------------------------ plain forms
def _slots(table, start, width):
    """Pool rows [n_seqs, width] of slots 0 .. width - 1 (those past a prompt's length are not used)."""
    t = torch.arange(width, device="cuda")
    if table is not None:
        return table.long()[:, t // PAGE] * PAGE + t % PAGE
    return start.long()[:, None] + t


def _scores(s):
    """Scores [n_seqs, kv_heads, nodes, group, slots] of all nodes, what each sees, and where the rows sit."""
    n, hkv, hq, d = s["ctx_len"].numel(), s["k"].shape[1], s["q"].shape[1], s["q"].shape[2]
    m, t = s["max_nodes"], s["max_len"]
    ctx, first = s["ctx_len"].long(), s["row_start"].long()
    count = first[1:] - first[:-1]
    node = torch.arange(m, device="cuda")
    slot = torch.arange(t, device="cuda")
    real = node < count[:, None]                                                      # [n, m]
    row = torch.where(real, first[:-1, None] + node, first[:-1, None])
    at = torch.minimum(_slots(s.get("page_table"), s.get("ctx_start"), t), torch.tensor(s["k"].shape[0] - 1, device="cuda"))
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
    qf = s["q"][row].float().view(n, m, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, d)
    kf = s["k"][at].float().permute(0, 2, 3, 1)                                       # [n, hkv, d, t]
    x = torch.matmul(qf, kf).view(n, hkv, m, hq // hkv, t) * s["scale"]
    return x, seen, real, row, at


def _tree_plain(s):
    x, seen, real, row, at = _scores(s)
    n, hkv, m, g, t = x.shape
    x = x.masked_fill(~seen[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(seen.any(-1)[:, None, :, None, None], top, torch.zeros_like(top))
    x = torch.exp(x - top)
    total = x.sum(-1)                                                                 # [n, hkv, m, g]
    inside = torch.arange(t, device="cuda") < (s["ctx_len"].long() + (s["row_start"][1:] - s["row_start"][:-1]).long())[:, None]
    vf = torch.where(inside[:, :, None, None], s["v"][at].float(), torch.zeros((), device="cuda")).permute(0, 2, 1, 3)
    o = torch.matmul(x.view(n, hkv, m * g, t), vf).view(n, hkv, m, g, -1)
    o = torch.where(seen.any(-1)[:, None, :, None, None], o / total[..., None], torch.zeros((), device="cuda"))
    lse = torch.log(total) + top[..., 0]
    out = torch.zeros((s["q"].shape[0], hkv * g, vf.shape[-1]), dtype=s["q"].dtype, device="cuda")
    out[row[real]] = o.permute(0, 2, 1, 3, 4).reshape(n, m, hkv * g, -1)[real].to(s["q"].dtype)
    all_lse = torch.zeros((s["q"].shape[0], hkv * g), device="cuda")
    all_lse[row[real]] = lse.permute(0, 2, 1, 3).reshape(n, m, hkv * g)[real]
    return {"out": out, "lse": all_lse}


def _weights_plain(s):
    x, seen, real, row, at = _scores(s)
    n, hkv, m, g, t = x.shape
    seen = seen & (s["use"][row] != 0)[:, :, None]
    lse = s["lse"][row].view(n, m, hkv, g).permute(0, 2, 1, 3)
    p = torch.exp(x - lse[..., None]).masked_fill(~seen[:, None, :, None, :], 0.0)
    inside = torch.arange(t, device="cuda") < (s["ctx_len"].long() + (s["row_start"][1:] - s["row_start"][:-1]).long())[:, None]
    out = torch.where(inside[:, None, :], DECAY * s["weights"] + p.sum((2, 3)), torch.zeros((), device="cuda"))
    return {"weights": out}


def _select_plain(weights, length, budget, sink, recent):
    n, h, t = weights.shape
    slot = torch.arange(t, device="cuda")
    length = length.long()[:, None]
    w = torch.where(torch.isnan(weights), torch.full_like(weights, -math.inf), weights)
    always = (slot < sink) | (slot >= length - recent)
    tier = torch.where(slot < length, 1 + always.long(), 0)[:, None, :].expand(n, h, t)
    by_weight = torch.sort(w, dim=-1, descending=True, stable=True).indices
    order = torch.sort(torch.gather(tier, 2, by_weight), dim=-1, descending=True, stable=True).indices
    best = torch.gather(by_weight, 2, order)[:, :, :budget]
    count = torch.minimum(length[:, 0], torch.tensor(budget, device="cuda"))
    place = torch.arange(best.shape[2], device="cuda")
    best = torch.where(place < count[:, None, None], best, torch.tensor(t, device="cuda")).sort(-1).values
    keep = torch.full((n, h, budget), -1, dtype=torch.int32, device="cuda")
    keep[:, :, :best.shape[2]] = torch.where(best < t, best, torch.tensor(-1, device="cuda")).to(torch.int32)
    return keep, count.to(torch.int32)


def _compact_plain(s):
    keep, count = s["keep"].long(), s["count"].long()
    n, h, m = keep.shape
    valid = (torch.arange(m, device="cuda") < count[:, None])[:, None, :].expand(n, h, m)
    src = torch.gather(_slots(s.get("page_table"), s.get("ctx_start"), s["max_len"])[:, None, :].expand(n, h, -1), 2, keep.clamp(min=0))
    dst = _slots(s.get("dst_page_table"), s.get("dst_start"), m)[:, None, :].expand(n, h, m)
    head = torch.arange(h, device="cuda")[None, :, None].expand(n, h, m)
    k, v, w = s["k"], s["v"], s["weights_out"]
    k[dst[valid], head[valid]] = k[src[valid], head[valid]]
    v[dst[valid], head[valid]] = v[src[valid], head[valid]]
    w[:, :, :m] = torch.where(valid, torch.gather(s["weights"], 2, keep.clamp(min=0)), w[:, :, :m])
    return {"k": k, "v": v, "weights": w}


DECAY = 0.875


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2601_11553_b200 import percache as pc
        stream = torch.cuda.current_stream().cuda_stream
        if op == "tree":
            pc.tree_attention(s["q"], s["k"], s["v"], s["out"], s["lse"], ctx_len=s["ctx_len"], row_start=s["row_start"],
                              mask=s["mask"], page_table=s.get("page_table"), ctx_start=s.get("ctx_start"),
                              max_nodes=s["max_nodes"], max_len=s["max_len"], scale=s["scale"], workspace=s["workspace"],
                              stream=stream)
            return {"out": s["out"], "lse": s["lse"]}
        if op == "weights":
            pc.attention_weights(s["q"], s["k"], s["lse"], s["weights"], s["weights_out"], ctx_len=s["ctx_len"],
                                 row_start=s["row_start"], mask=s["mask"], use=s["use"], page_table=s.get("page_table"),
                                 ctx_start=s.get("ctx_start"), max_nodes=s["max_nodes"], max_len=s["max_len"],
                                 scale=s["scale"], decay=DECAY, workspace=s["workspace"], stream=stream)
            return {"weights": s["weights_out"]}
        if op == "select":
            pc.select_slots(s["weights"], s["length"], s["keep"], s["count"], sink=s["case"]["sink"],
                            recent=s["case"]["recent"], max_len=s["max_len"], stream=stream)
            return {"keep": s["keep"], "count": s["count"]}
        pc.compact_slots(s["k"], s["v"], s["keep"], s["count"], weights=s["weights"], weights_out=s["weights_out"],
                         page_table=s.get("page_table"), ctx_start=s.get("ctx_start"),
                         dst_page_table=s.get("dst_page_table"), dst_start=s.get("dst_start"), max_len=s["max_len"],
                         stream=stream)
        return {"k": s["k"], "v": s["v"], "weights": s["weights_out"]}
    if op == "tree":
        return _tree_plain(s)
    if op == "weights":
        return _weights_plain(s)
    if op == "select":
        keep, count = _select_plain(s["weights"], s["length"], s["case"]["budget"], s["case"]["sink"], s["case"]["recent"])
        return {"keep": keep, "count": count}
    return _compact_plain(s)


# ------------------------------------------------------------------------------------------------------------ least work
def work(case):
    ctx, nodes = _lengths(case)
    hkv, hq, d = case["kv_heads"], case["q_heads"], case["head_dim"]
    lens = [a + b for a, b in zip(ctx, nodes)]
    table = sum(-(-t // PAGE) for t in lens) * 4 if case["paged"] else 4 * case["n_seqs"]
    if case["op"] == "tree":
        return {"bytes": sum(lens) * hkv * d * 4 + sum(nodes) * hq * (4 * d + 4) + table,
                "flops": 4 * d * hq * sum(m * (t + 1) for m, t in zip(nodes, ctx))}
    if case["op"] == "weights":
        used = [sum(_used(case, i) for i in range(m)) for m in nodes]
        return {"bytes": sum(lens) * hkv * (2 * d + 8) + sum(used) * hq * (2 * d + 4) + table,
                "flops": 2 * d * hq * sum(m * (t + 1) for m, t in zip(used, ctx))}
    kept = sum(min(t, case["budget"]) for t in ctx)
    if case["op"] == "select":
        return {"bytes": sum(ctx) * hkv * 4 + case["n_seqs"] * hkv * case["budget"] * 4, "flops": 0}
    return {"bytes": kept * hkv * (8 * d + 12) + table, "flops": 0}


# ------------------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """Prompt by prompt, straight from the definitions."""
    if case["op"] in ("select", "compact"):
        return None                    # whole numbers, and values that are only moved
    s = prepare(case, seed)
    ctx, nodes = _lengths(case)
    hkv, hq, d = case["kv_heads"], case["q_heads"], case["head_dim"]
    g = hq // hkv
    out = torch.zeros((sum(nodes), hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((sum(nodes), hq), dtype=torch.float64, device="cuda")
    if case["op"] == "weights":
        weights = torch.zeros(s["weights"].shape, dtype=torch.float64, device="cuda")
        use = s["use"].cpu().tolist()
    r0 = 0
    for b in range(case["n_seqs"]):
        c, m = ctx[b], nodes[b]
        t = c + m
        if case["paged"]:
            rows = (s["page_table"][b].long()[:, None] * PAGE + torch.arange(PAGE, device="cuda")).reshape(-1)[:t]
        else:
            rows = torch.arange(t, device="cuda") + int(s["ctx_start"][b])
        hidden = torch.zeros((m, t), dtype=torch.bool)
        if s["mask"] is None:
            hidden[:, c:] = torch.ones((m, m)).triu(1).bool()
        else:
            words = s["mask"][r0:r0 + m].cpu().tolist()
            for i in range(m):
                for j in range(m):
                    hidden[i, c + j] = not (words[i][j // 64] >> (j % 64)) & 1
        hidden = hidden.cuda()
        for h in range(hkv):
            k = s["k"][rows, h].double()
            v = s["v"][rows, h].double()
            for q in range(h * g, (h + 1) * g):
                x = (s["q"][r0:r0 + m, q].double() @ k.T) * s["scale"]
                x[hidden] = -math.inf
                if case["op"] == "tree":
                    z = torch.logsumexp(x, -1)
                    lse[r0:r0 + m, q] = z
                    out[r0:r0 + m, q] = torch.softmax(x, -1) @ v
                else:
                    for i in range(m):
                        if use[r0 + i]:
                            weights[b, h, :t] += torch.exp(x[i] - s["lse"][r0 + i, q].double())
        if case["op"] == "weights":
            weights[b, :, :t] += DECAY * s["weights"][b, :, :t].double()
        r0 += m
    return {"out": out, "lse": lse} if case["op"] == "tree" else {"weights": weights}
