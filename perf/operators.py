"""The decode-side operators whose speed this library is kept to, as a user's program calls them.

Four operators that one token of generation needs beside the products with compressed weights: attention of one new
token over a paged key-value cache (`attn`), the write of new tokens into that cache (`append`), eviction from it by
accumulated attention weight (`evict`), and products with 4-bit weights (`q4`).  Where `own` is false `run` computes
them in elementary torch operations in 32 bits; where it is true it calls the library.

The calls give their results in buffers of their own (`new_lengths` and so on) rather than in place, so that a state can
be run again; what they write into the cache's pages is the same each time.
"""
import math

import torch

own = False

# Attention heads of the two models whose linear layers the library is built around: q heads, kv heads, head width
OPT66B_HEADS = (72, 72, 128)
LLAMA2_70B_HEADS = (64, 8, 128)


def _attn(batch, heads, length, page, dtype="f16", ragged=False, weights=False, mask=False):
    return {"op": "attn", "batch": batch, "q_heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "length": length,
            "page": page, "dtype": dtype, "ragged": ragged, "weights": weights, "mask": mask}


def _evict(batch, kv_heads, dim, length, budget, recent, page, dtype="f16", ragged=False):
    return {"op": "evict", "batch": batch, "kv_heads": kv_heads, "dim": dim, "length": length, "budget": budget,
            "recent": recent, "page": page, "dtype": dtype, "ragged": ragged}


def _append(batch, kv_heads, dim, tokens, length, page, dtype="f16", ragged=False):
    return {"op": "append", "batch": batch, "kv_heads": kv_heads, "dim": dim, "tokens": tokens, "length": length,
            "page": page, "dtype": dtype, "ragged": ragged}


def _q4(rows, cols, nb, group, zeros, dtype="f16"):
    return {"op": "q4", "rows": rows, "cols": cols, "nb": nb, "group": group, "zeros": zeros, "dtype": dtype}


def listed():
    return [
        # One Llama2-70B layer, one sequence, the first tokens after a short prompt: latency and launches count.
        {"name": "attn_llama2_70b_short", **_attn(1, LLAMA2_70B_HEADS, 131, 16)},
        # OPT-66B, whose heads share nothing, over its whole context of 2048 for eight sequences of different lengths,
        # one of them not begun; the weights that eviction goes by are summed up on the way.
        {"name": "attn_opt66b_batch", **_attn(8, OPT66B_HEADS, 2048, 16, ragged=True, weights=True)},
        # One very long sequence: all parallelism comes from splitting it.
        {"name": "attn_llama2_70b_long", **_attn(1, LLAMA2_70B_HEADS, 131072, 64)},
        # A server's batch of narrow bfloat16 heads, ragged, left-padded, one row hidden altogether.
        {"name": "attn_ragged_bf16", **_attn(48, (32, 8, 64), 4001, 32, "bf16", ragged=True, weights=True, mask=True)},
        # Eviction as it comes at every token once a cache is full: one token over the budget in every sequence.
        {"name": "evict_llama2_70b_step", **_evict(4, 8, 128, 2049, 2048, 256, 16)},
        # Eviction after prompts: ragged, some sequences below the budget.
        {"name": "evict_ragged_bf16", **_evict(16, 8, 128, 16000, 4096, 513, 64, "bf16", ragged=True)},
        # One new token for each of a batch of sequences.
        {"name": "append_llama2_70b_token", **_append(32, 8, 128, 1, 4000, 16)},
        # Prompts of OPT-66B written into the cache, ragged: not every sequence brings all the tokens.
        {"name": "append_opt66b_prompt", **_append(4, 72, 128, 1777, 200, 16, ragged=True)},
        # The smallest product: the key projection of a Llama2-70B layer, one token.
        {"name": "q4_llama2_70b_k", **_q4(1024, 8192, 1, 128, False)},
        # One token against the down projection.
        {"name": "q4_llama2_70b_down", **_q4(8192, 28672, 1, 128, False)},
        # A full small batch against the gate projection, narrow groups with zero points.
        {"name": "q4_llama2_70b_gate16", **_q4(28672, 8192, 16, 64, True)},
        # A few bfloat16 tokens against an odd-sized matrix: the last group is partial, rows end inside bytes.
        {"name": "q4_odd_bf16", **_q4(5003, 3171, 3, 32, True, "bf16")},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, sizes from the smallest listed ones to the largest, round and odd."""
    op = rng.choice(["attn", "attn", "attn", "evict", "append", "q4", "q4", "q4"])
    dtype = rng.choice(["f16", "bf16"])
    if op == "q4":
        while True:
            rows, cols = _log_uniform(rng, 512, 36864), _log_uniform(rng, 512, 36864)
            if rng.random() < 0.6:
                rows, cols = max(64, rows // 64 * 64), max(64, cols // 64 * 64)
            if rows * cols <= 28672 * 8192 and 3072 not in (rows, cols):
                break
        return _q4(rows, cols, rng.choice([1, 1, rng.randint(2, 16)]), rng.choice([32, 64, 128, 128, 256]), rng.random() < 0.5, dtype)
    page = rng.choice([8, 16, 16, 32, 64, 128, 256])
    dim = rng.choice([64, 80, 96, 128, 128, 128, 256])
    if op == "attn":
        while True:
            kv = rng.choice([1, 2, 4, 8, 8, 16, 32, 72])
            group = rng.choice([1, 1, 2, 4, 7, 8, 8, 16])
            batch, length = _log_uniform(rng, 1, 64), _log_uniform(rng, 1, 131072)
            if kv * group <= 128 and batch * length * kv * dim <= 131072 * 8 * 128 and length != 3072:
                break
        return _attn(batch, (kv * group, kv, dim), length, page, dtype, rng.random() < 0.6, rng.random() < 0.4, rng.random() < 0.3)
    kv = rng.choice([1, 4, 8, 8, 16, 32, 72])
    ragged = rng.random() < 0.5
    if op == "evict":
        while True:
            batch, length = _log_uniform(rng, 1, 32), _log_uniform(rng, 64, 32768)
            if batch * length * kv * dim <= 16 * 16000 * 8 * 128 and length != 3072:
                break
        budget = max(1, int(length * rng.choice([0.25, 0.5, 0.75, 0.9, 1 - 1.0 / length])))
        budget += budget == 3072
        return _evict(batch, kv, dim, length, budget, int(budget * rng.uniform(0, 0.5)), page, dtype, ragged)
    while True:
        batch, tokens = _log_uniform(rng, 1, 64), rng.choice([1, 1, _log_uniform(rng, 2, 4096)])
        length = rng.randint(0, 4096)
        if batch * (tokens + length) * kv * dim <= 4 * 1977 * 72 * 128 and 3072 not in (tokens, length):
            break
    return _append(batch, kv, dim, tokens, length, page, dtype, ragged)


# ---------------------------------------------------------------- sizes that follow from a case

def _spread(most, batch, ragged):
    """What each sequence of the batch has: `most`, or a spread from nothing to `most` that favours the short."""
    if not ragged or batch == 1:
        return [most] * batch
    return [int(round(most * (i / (batch - 1)) ** 1.5)) for i in range(batch)]


def _hidden(case):
    """(first visible slot of each sequence): an eighth of its length is padding on the left; the second sequence is all padding."""
    lengths = _spread(case["length"], case["batch"], case["ragged"])
    if not case["mask"]:
        return [0] * len(lengths)
    return [n if i == 1 else n // 8 for i, n in enumerate(lengths)]


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 17)


def _dtype(case):
    return torch.float16 if case["dtype"] == "f16" else torch.bfloat16


def _order(values, gen):
    """The sequences of a batch come in any order."""
    at = torch.randperm(len(values), generator=gen, device="cuda")
    return torch.tensor(values, dtype=torch.int32, device="cuda")[at], at


def _pool(case, need, gen):
    """A pool of pages in which sequences hold theirs at random places, some pages free: keys, values and the table of pages.
    Entries of the table past a sequence's pages are -1, as for pages not given out."""
    batch, page = case["batch"], case["page"]
    most = max(1, -(-max(need) // page))
    count = sum(-(-n // page) for n in need)
    table = torch.full((batch, most), -1, dtype=torch.int32, device="cuda")
    given = torch.randperm(count + 3, generator=gen, device="cuda")[:count].to(torch.int32)
    have = torch.tensor([-(-n // page) for n in need], device="cuda")
    table[torch.arange(most, device="cuda") < have[:, None]] = given
    shape = (count + 3, case["kv_heads"], page, case["dim"])
    k = torch.randn(shape, generator=gen, device="cuda", dtype=_dtype(case))
    v = torch.randn(shape, generator=gen, device="cuda", dtype=_dtype(case))
    return k, v, table


def _weights(case, capacity, gen):
    """Accumulated attention weights: a few large, most small, a fifth exactly zero (ties)."""
    shape = (case["batch"], case["kv_heads"], capacity)
    u = torch.rand(shape, generator=gen, device="cuda")
    return torch.where(u < 0.2, 0.0, -torch.log(1 - u) ** 3)


def _bits(visible):
    """Truth values [batch, slots] as 64-bit words, bit s & 63 of word s >> 6."""
    batch, slots = visible.shape
    words = torch.zeros((batch, -(-slots // 64) * 64), dtype=torch.int64, device="cuda")
    words[:, :slots] = visible
    return (words.view(batch, -1, 64) << torch.arange(64, device="cuda")).sum(-1)  # distinct bits: the sum is their union


def _attn_inputs(case, seed):
    gen = _generator(seed)
    need, at = _order(_spread(case["length"], case["batch"], case["ragged"]), gen)
    k, v, table = _pool(case, need.tolist(), gen)
    q = 2 * torch.randn((case["batch"], case["q_heads"], case["dim"]), generator=gen, device="cuda")
    s = {"lengths": need, "k": k, "v": v, "table": table, "q": q.to(_dtype(case)), "scale": case["dim"] ** -0.5,
         "capacity": table.shape[1] * case["page"], "max_len": case["length"], "weights": None, "visible": None}
    if case["weights"]:
        s["weights"] = _weights(case, s["capacity"], gen)
    if case["mask"]:
        first = torch.tensor(_hidden(case), device="cuda")[at]
        s["visible"] = torch.arange(s["capacity"], device="cuda") >= first[:, None]
    return s


def _evict_inputs(case, seed):
    gen = _generator(seed)
    need, _ = _order(_spread(case["length"], case["batch"], case["ragged"]), gen)
    k, v, table = _pool(case, need.tolist(), gen)
    capacity = table.shape[1] * case["page"]
    # A cache that has been evicted from before: as many tokens were seen again as it holds, the older half lies in any order.
    slot = torch.arange(capacity, device="cuda", dtype=torch.int32).expand(case["batch"], case["kv_heads"], capacity)
    half = (need // 2)[:, None, None]
    mixed = torch.rand(slot.shape, generator=gen, device="cuda").masked_fill(slot >= half, 2.0).argsort(-1).to(torch.int32)
    positions = torch.where(slot < half, 2 * mixed, slot + need[:, None, None]).to(torch.int32)
    return {"lengths": need, "seen": 2 * need, "k": k, "v": v, "table": table, "positions": positions, "capacity": capacity,
            "weights": _weights(case, capacity, gen), "budget": case["budget"], "recent": case["recent"], "max_len": case["length"]}


def _append_inputs(case, seed):
    gen = _generator(seed)
    batch, tokens, kv, dim = case["batch"], case["tokens"], case["kv_heads"], case["dim"]
    lengths, _ = _order(_spread(case["length"], batch, case["ragged"]), gen)
    counts = None
    if tokens > 1:
        counts, _ = _order([tokens - n for n in _spread(tokens - 1, batch, case["ragged"])] if case["ragged"] else [tokens] * batch, gen)
    k, v, table = _pool(case, [n + tokens for n in lengths.tolist()], gen)
    capacity = table.shape[1] * case["page"]
    new = torch.randn((2, batch, tokens, kv, dim), generator=gen, device="cuda", dtype=_dtype(case))
    return {"lengths": lengths, "seen": lengths + 5, "counts": counts, "k": k, "v": v, "table": table, "capacity": capacity,
            "new_k": new[0], "new_v": new[1], "weights": _weights(case, capacity, gen),
            "positions": torch.randint(0, 9999, (batch, kv, capacity), generator=gen, device="cuda", dtype=torch.int32)}


def _q4_inputs(case, seed):
    """A quantized weight as a checkpoint holds it: two codes a byte (the even column in the low half), a scale per row and
    group, whole zero points or none (then 8)."""
    gen = _generator(seed)
    rows, cols, groups = case["rows"], case["cols"], -(-case["cols"] // case["group"])
    codes = torch.randint(0, 256, (rows, (cols + 1) // 2), generator=gen, device="cuda", dtype=torch.uint8)
    scales = ((0.5 + torch.rand((rows, groups), generator=gen, device="cuda")) * 0.006).half()
    zeros = torch.randint(0, 16, (rows, groups), generator=gen, device="cuda", dtype=torch.uint8) if case["zeros"] else None
    x = torch.randn((case["nb"], cols), generator=gen, device="cuda").to(_dtype(case))
    return {"codes": codes, "scales": scales, "zeros": zeros, "x": x, "group": case["group"], "rows": rows, "cols": cols}


_INPUTS = {"attn": _attn_inputs, "evict": _evict_inputs, "append": _append_inputs, "q4": _q4_inputs}


def prepare(case, seed):
    """Inputs, the buffers that a program keeps from token to token, and the library's handles for them."""
    op = case["op"]
    s = {"op": op, **_INPUTS[op](case, seed)}
    if op == "q4":
        s["y"] = torch.empty((case["nb"], case["rows"]), dtype=torch.float32, device="cuda")
    else:
        s["new_lengths"], s["new_seen"] = torch.empty_like(s["lengths"]), torch.empty_like(s["lengths"])
        if s["weights"] is not None:
            s["new_weights"] = torch.zeros_like(s["weights"])
        if op == "evict":
            s["new_positions"] = torch.zeros_like(s["positions"])
        if op == "attn":
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    if own:
        import paper_2406_11674_amd as endor
        s["endor"] = endor
        if op == "q4":
            s["m"] = endor.q4_pack(s["codes"], s["scales"], s["zeros"], s["cols"], s["group"])
            del s["codes"]
        else:
            s["cache"] = endor.KVCache(s["k"], s["v"], s["table"])
        if op == "attn":
            s["scratch"] = s["cache"].attn_scratch(case["q_heads"], s["max_len"], weights=case["weights"])
            s["mask"] = _bits(s["visible"]) if case["mask"] else None
        if op == "evict":
            s["scratch"] = s["cache"].evict_scratch(s["budget"], s["max_len"])
    return s


# ---------------------------------------------------------------- one pass: the library's calls

def _run_own(s):
    op, endor = s["op"], s["endor"]
    if op == "q4":
        return endor.q4_gemm(s["m"], s["x"], Y=s["y"])
    if op == "attn":
        endor.attn_decode(s["cache"], s["q"], s["lengths"], max_len=s["max_len"], mask=s["mask"], scale=s["scale"],
                          weights=s["weights"], new_weights=s.get("new_weights"), out=s["out"], lse=s["lse"], scratch=s["scratch"])
        return {"out": s["out"], "lse": s["lse"], "weights": s.get("new_weights")}
    if op == "evict":
        endor.kv_evict(s["cache"], s["lengths"], s["seen"], s["weights"], s["positions"], s["budget"], s["recent"],
                       max_len=s["max_len"], new_lengths=s["new_lengths"], new_weights=s["new_weights"],
                       new_positions=s["new_positions"], scratch=s["scratch"])
        return {"k": s["k"], "v": s["v"], "lengths": s["new_lengths"], "weights": s["new_weights"], "positions": s["new_positions"]}
    endor.kv_append(s["cache"], s["new_k"], s["new_v"], s["lengths"], s["seen"], counts=s["counts"], weights=s["weights"],
                    positions=s["positions"], new_lengths=s["new_lengths"], new_seen=s["new_seen"])
    return {"k": s["k"], "v": s["v"], "lengths": s["new_lengths"], "seen": s["new_seen"], "weights": s["weights"],
            "positions": s["positions"]}


# ---------------------------------------------------------------- one pass: plain torch

def _gather(pages, table):
    """A cache's tokens in order, in 32 bits: [batch, kv head, slot, dim]."""
    got = pages[table.clamp(min=0).long()]
    batch, count, heads, page, dim = got.shape
    return got.permute(0, 2, 1, 3, 4).reshape(batch, heads, count * page, dim).float()


def _plain_attn(s):
    q = s["q"].float()
    batch, q_heads, dim = q.shape
    kv_heads, slots = s["k"].shape[1], s["capacity"]
    slot = torch.arange(slots, device="cuda")
    live = slot < s["lengths"][:, None]
    if s["visible"] is not None:
        live = live & s["visible"]
    live = live[:, None, None, :]
    qt = q.view(batch, kv_heads, q_heads // kv_heads, dim).transpose(2, 3).contiguous()
    scores = (torch.matmul(_gather(s["k"], s["table"]), qt) * s["scale"]).transpose(2, 3).contiguous()
    scores = scores.masked_fill(~live, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - top.masked_fill(top == -math.inf, 0.0))
    total = e.sum(-1, keepdim=True)
    p = e / total.masked_fill(total == 0, 1.0)
    v = _gather(s["v"], s["table"]).masked_fill_(~live.transpose(2, 3), 0.0)
    out = torch.matmul(p, v).view(batch, q_heads, dim).to(s["q"].dtype)
    lse = (top + torch.log(total)).view(batch, q_heads)
    new = None
    if s["weights"] is not None:
        held = (slot < s["lengths"][:, None])[:, None, :]
        new = torch.where(held, s["weights"] + p.sum(2), s["new_weights"])
    return {"out": out, "lse": lse, "weights": new}


def _places(s, slots):
    """(page, slot in the page) of slots [batch, kv head, n]."""
    page = s["k"].shape[2]
    rows = s["table"].long()[:, None, :].expand(-1, slots.shape[1], -1)
    return rows.gather(2, slots // page), slots % page


def _plain_evict(s):
    batch, heads, slots = s["weights"].shape
    slot = torch.arange(slots, device="cuda").expand(batch, heads, slots)
    length = s["lengths"].long()[:, None, None]
    live = slot < length
    after = torch.minimum(length, torch.full_like(length, s["budget"]))
    key = s["weights"].masked_fill(s["weights"].isnan(), -math.inf)
    key = key.masked_fill(s["positions"] >= (s["seen"][:, None, None] - s["recent"]), math.inf)
    order = key.masked_fill(~live, -math.inf)
    # slots past the length are behind all others, whatever those weigh
    by = torch.sort(order, dim=-1, descending=True, stable=True).indices
    by = by.gather(-1, torch.sort((~live).gather(-1, by).to(torch.uint8), dim=-1, stable=True).indices)
    rank = torch.empty_like(by).scatter_(-1, by, slot)
    keep = live & (rank < after)
    hole, mover = ~keep & (slot < after), keep & (slot >= after)
    # the i-th hole takes the i-th mover
    holes = torch.sort((~hole).to(torch.uint8), dim=-1, stable=True).indices
    movers = torch.sort((~mover).to(torch.uint8), dim=-1, stable=True).indices
    come = slot < hole.sum(-1, keepdim=True)
    source = slot.clone().scatter_(-1, holes, torch.where(come, movers, holes))
    held = slot < after
    weights = torch.where(held, s["weights"].gather(-1, source), s["new_weights"])
    positions = torch.where(held, s["positions"].gather(-1, source), s["new_positions"])
    which = come.nonzero(as_tuple=True)
    to, off = (x[which] for x in _places(s, holes))
    page, at = (x[which] for x in _places(s, movers))
    for pages in (s["k"], s["v"]):
        pages[to, which[1], off] = pages[page, which[1], at]
    return {"k": s["k"], "v": s["v"], "lengths": after.view(-1).to(torch.int32), "weights": weights, "positions": positions}


def _plain_append(s):
    batch, tokens, heads, _ = s["new_k"].shape
    counts = s["counts"] if s["counts"] is not None else torch.full_like(s["lengths"], tokens)
    t = torch.arange(tokens, device="cuda").expand(batch, tokens)
    which = (t < counts[:, None]).nonzero(as_tuple=True)
    slots = (s["lengths"].long()[:, None] + t)[:, None, :]
    page, at = (x[:, 0][which] for x in _places(s, slots))
    s["k"][page, :, at] = s["new_k"][which]
    s["v"][page, :, at] = s["new_v"][which]
    slots = slots[:, 0][which]
    s["weights"][which[0], :, slots] = 0.0
    s["positions"][which[0], :, slots] = (s["seen"][:, None] + t)[which].to(torch.int32)[:, None]
    return {"k": s["k"], "v": s["v"], "lengths": s["lengths"] + counts, "seen": s["seen"] + counts, "weights": s["weights"],
            "positions": s["positions"]}


def _plain_q4(s):
    codes = torch.stack((s["codes"] & 15, s["codes"] >> 4), dim=-1).view(s["rows"], -1)[:, :s["cols"]].float()
    wide = lambda t: t.float().repeat_interleave(s["group"], dim=1)[:, :s["cols"]]  # noqa: E731
    w = (codes - (8.0 if s["zeros"] is None else wide(s["zeros"]))) * wide(s["scales"])
    return torch.matmul(s["x"].float(), w.t())


_PLAIN = {"attn": _plain_attn, "evict": _plain_evict, "append": _plain_append, "q4": _plain_q4}


def run(state):
    return _run_own(state) if "endor" in state else _PLAIN[state["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    op = case["op"]
    if op == "q4":
        rows, cols, nb = case["rows"], case["cols"], case["nb"]
        groups = -(-cols // case["group"])
        return {"bytes": rows * cols / 2 + rows * groups * (3 if case["zeros"] else 2) + nb * (2 * cols + 4 * rows),
                "flops": 2.0 * nb * rows * cols}
    batch, heads, dim = case["batch"], case["kv_heads"], case["dim"]
    token = 4 * dim * heads  # bytes of one token's keys and values
    lengths = _spread(case["length"], batch, case["ragged"])
    if op == "attn":
        seen = sum(n - h for n, h in zip(lengths, _hidden(case)))
        return {"bytes": seen * token + batch * case["q_heads"] * (4 * dim + 4) + (8 * heads * sum(lengths) if case["weights"] else 0),
                "flops": 4.0 * seen * case["q_heads"] * dim}
    if op == "evict":
        budget, recent = case["budget"], case["recent"]
        kept, moved = sum(min(n, budget) for n in lengths), 0.0
        for n in lengths:
            if n > budget:  # the newest tokens, and a share of the others that lie past the budget
                moved += min(recent, n - budget) + (max(0, n - recent - budget) * (budget - recent) / (n - recent) if n > recent else 0)
        return {"bytes": heads * 8 * (sum(lengths) + kept) + 2 * moved * token, "flops": 0}
    tokens = case["tokens"]
    count = sum(tokens - n for n in _spread(tokens - 1, batch, case["ragged"])) if tokens > 1 and case["ragged"] else batch * tokens
    return {"bytes": count * (2 * token + 8 * heads) + 16 * batch, "flops": 0}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    """From each operator's definition, sequence by sequence, in 64 bits; nothing for values that are only moved."""
    if case["op"] not in ("attn", "q4"):
        return None
    s = _INPUTS[case["op"]](case, seed)
    if case["op"] == "q4":
        y = torch.zeros((case["nb"], case["rows"]), dtype=torch.float64, device="cuda")
        x = s["x"].double()
        for g in range(s["scales"].shape[1]):
            lo, hi = g * s["group"], min(s["cols"], (g + 1) * s["group"])
            at = torch.arange(lo, hi, device="cuda")
            c = ((s["codes"][:, at // 2] >> (4 * (at % 2)).to(torch.uint8)) & 15).double()
            z = 8.0 if s["zeros"] is None else s["zeros"][:, g:g + 1].double()
            y += (x[:, lo:hi] @ (c - z).t().contiguous()) * s["scales"][:, g].double()
        return y
    page, heads = case["page"], case["kv_heads"]
    group = case["q_heads"] // heads
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    new = torch.zeros_like(s["weights"], dtype=torch.float64) if case["weights"] else None
    for b, n in enumerate(s["lengths"].tolist()):
        slots = torch.arange(n, device="cuda")
        if case["weights"]:
            new[b, :, :n] = s["weights"][b, :, :n].double()
        if case["mask"]:
            slots = slots[s["visible"][b, :n]]
        if slots.numel() == 0:
            continue
        at, off = s["table"][b].long()[slots // page], slots % page
        for h in range(heads):
            k, v = s["k"][at, h, off].double(), s["v"][at, h, off].double()
            mine = slice(h * group, (h + 1) * group)
            logits = s["q"][b, mine].double() @ k.t().contiguous() * s["scale"]
            lse[b, mine] = torch.logsumexp(logits, -1)
            p = torch.softmax(logits, -1)
            out[b, mine] = p @ v
            if case["weights"]:
                new[b, h, slots] += p.sum(0)
    return {"out": out, "lse": lse, "weights": new}
