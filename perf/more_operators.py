"""Cases and plain forms of the operators for a paged 16-bit key-value cache and beam search over it: block tables and
slot maps from request lengths, rows stored by slot, attention of one new token over pages, and the selection of beams.

Head counts, vocabularies and lengths are those of the workloads in ``paper_2604_04722_b200/synth.py`` (SmolLM-135M/360M/
1.7B-shaped layers), besides one grouped-query shape with 128 channels.  ``own`` selects between the plain forms below and
the framework's entry points.
"""
import math

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    att = dict(op="attn", ragged=False, order="slots")
    step = dict(op="step", beams=1, joins=0, prompt=0)
    return [
        # one user of the smallest model on a short prompt: latency
        dict(att, name="attn_cfg1_1x512", batch=1, q_heads=9, kv_heads=3, head_dim=64, ctx=512, page=16, dtype="fp16"),
        # one user with a long document: a few heads, split over the length
        dict(att, name="attn_1x32768", batch=1, q_heads=15, kv_heads=5, head_dim=64, ctx=32768, page=16, dtype="fp16"),
        # a ragged batch of grouped-query requests, one of them a padding row, odd lengths
        dict(att, name="attn_cfg3_8x4001_ragged", batch=8, q_heads=15, kv_heads=5, head_dim=64, ctx=4001, page=16,
             dtype="bf16", ragged=True),
        # a large batch on the largest model, one query head per KV head: throughput
        dict(att, name="attn_cfg4_16x8192", batch=16, q_heads=32, kv_heads=32, head_dim=64, ctx=8192, page=64, dtype="fp16"),
        # a serving batch of grouped queries over 128 channels, pages kept head by head
        dict(att, name="attn_gqa_64x4096_ragged", batch=64, q_heads=32, kv_heads=8, head_dim=128, ctx=4096, page=16,
             dtype="bf16", ragged=True, order="heads"),
        # a decode step of 64 requests with four beams each; requests that come with their prompts beside others that go on
        dict(step, name="step_256x4096_beams", batch=256, ctx=4096, page=16, spare=8192, beams=4),
        dict(step, name="step_96x2000_joins", batch=96, ctx=2000, page=32, spare=4096, joins=24, prompt=1500),
        # the rows of one beam step; the rows of a prompt batch
        dict(op="append", name="append_16x5_beams", tokens=16, kv_heads=5, head_dim=64, page=16, pages=4096, copies=8, dtype="fp16"),
        dict(op="append", name="append_16001x32", tokens=16001, kv_heads=32, head_dim=64, page=64, pages=512, copies=0, dtype="bf16"),
        # one request with four beams; a batch of them in 32 bits; many, over an odd vocabulary
        dict(op="select", name="select_1x4", batch=1, beams=4, vocab=49152, dtype="fp16", ended=False, first=False),
        dict(op="select", name="select_16x8_fp32", batch=16, beams=8, vocab=49152, dtype="fp32", ended=True, first=False),
        dict(op="select", name="select_64x16_odd", batch=64, beams=16, vocab=32003, dtype="bf16", ended=True, first=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attn", "attn", "step", "append", "select"])
    if op == "attn":
        kv_heads, group = rng.choice([(3, 3), (5, 3), (32, 1), (8, 4), (1, 1), (2, 8), (1, 12), (4, 7)])
        ctx, batch, D = _log_int(rng, 1, 32768), _log_int(rng, 1, 128), rng.choice([64, 64, 128])
        while batch * kv_heads * ctx * D > 16 * 32 * 8192 * 64:
            batch, ctx = max(1, batch // 2), ctx if batch > 1 else ctx // 2
        return dict(op=op, batch=batch, q_heads=kv_heads * group, kv_heads=kv_heads, head_dim=D, ctx=ctx,
                    page=rng.choice([1, 8, 16, 16, 24, 32, 64, 128]), dtype=rng.choice(["fp16", "bf16"]),
                    ragged=rng.random() < 0.6, order=rng.choice(["slots", "heads"]))
    if op == "step":
        beams = rng.choice([1, 1, 2, 4, 5, 8])
        batch = beams * _log_int(rng, 1, 256 // beams)
        joins = rng.randint(0, batch // 4) if beams == 1 else 0
        return dict(op=op, batch=batch, ctx=_log_int(rng, 1, 4096), page=rng.choice([8, 16, 16, 32, 64]),
                    spare=_log_int(rng, 1024, 16384), beams=beams, joins=joins, prompt=_log_int(rng, 1, 1500) if joins else 0)
    if op == "append":
        c = dict(op=op, tokens=_log_int(rng, 1, 16384), kv_heads=rng.choice([1, 3, 5, 8, 32]), head_dim=rng.choice([64, 64, 128]),
                 page=rng.choice([8, 16, 24, 64]), copies=rng.choice([0, 0, rng.randint(1, 64)]), dtype=rng.choice(["fp16", "bf16"]))
        while c["tokens"] * c["kv_heads"] * c["head_dim"] > 16000 * 32 * 64:
            c["tokens"] //= 2
        c["pages"] = -(-c["tokens"] * 5 // (4 * c["page"])) + 2 * c["copies"] + 16
        return c
    beams = rng.randint(1, 16)
    c = dict(op=op, batch=_log_int(rng, 1, 64), beams=beams, vocab=_log_int(rng, 1000, 60000),
             dtype=rng.choice(["fp16", "bf16", "fp32"]), ended=rng.random() < 0.5, first=rng.random() < 0.2)
    while c["batch"] * beams * c["vocab"] * (2 if c["dtype"] == "fp32" else 1) > 64 * 16 * 32003:
        c["batch"] = max(1, c["batch"] // 2)
    return c


def _lens(case):
    """Cached tokens per row: all ``ctx``, or from about half of it up to ``ctx`` and one padding row."""
    n, B = case["ctx"], case["batch"]
    if not case["ragged"]:
        return [n] * B
    return [0 if b == B - 2 and B > 3 else n - b * 7919 % (n // 2 + 1) for b in range(B)]


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _pages(n_pages, case, g):
    """Keys or values of a cache: [pages][slots][heads][channels], kept slot by slot or head by head; four channels of a
    head are eight times as large."""
    H, D, page = case["kv_heads"], case["head_dim"], case["page"]
    scale = torch.ones(H, D, device="cuda")
    scale.scatter_(1, torch.rand(H, D, generator=g, device="cuda").argsort(dim=1)[:, :4], 8.0)
    heads_first = case.get("order") == "heads"
    shape, scale = ((n_pages, H, page, D), scale[:, None]) if heads_first else ((n_pages, page, H, D), scale)
    out = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda")
    for i in range(0, n_pages, 4096):
        part = out[i:i + 4096]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * scale)
    return out.transpose(1, 2) if heads_first else out


def _attn_inputs(case, seed):
    g = _gen(seed)
    B, page, lens = case["batch"], case["page"], _lens(case)
    width = -(-case["ctx"] // page)
    used = sum(-(-n // page) for n in lens)
    n_pages = used + used // 8 + 1
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    tables = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(lens):
        k = -(-n // page)
        tables[b, :k] = order[at:at + k]
        at += k
    x = {"K": _pages(n_pages, case, g), "V": _pages(n_pages, case, g), "tables": tables}
    x["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    x["Q"] = torch.randn((B, case["q_heads"], case["head_dim"]), generator=g, device="cuda").to(DTYPES[case["dtype"]])
    return x


def _step_inputs(case, seed):
    """Requests of ``beams`` rows: the first half of a request's tokens is its prompt, whose full pages its rows share."""
    g = _gen(seed)
    B, W, n, page = case["batch"], case["beams"], case["ctx"], case["page"]
    req = torch.arange(B, device="cuda") // W
    lens = (n - (torch.rand(B, generator=g, device="cuda") * (n // 2 + 1)).long()).clamp(min=0)
    lens = lens[req * W]                                # the beams of a request are as long as each other
    width = -(-(n + case["prompt"] + 1) // page)
    shared = torch.where(torch.tensor(W > 1, device="cuda"), lens // 2 // page, 0)
    col = torch.arange(width, device="cuda")
    listed_ = col < -(-lens // page)[:, None]
    mine = listed_ & ((col >= shared[:, None]) | (torch.arange(B, device="cuda") % W == 0)[:, None])
    n_pages = int(mine.sum()) + case["spare"] + B + (B * case["prompt"]) // page
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    place = (mine.flatten().cumsum(0) - 1).clamp(min=0).reshape(B, width)
    place = torch.where(mine, place, place[req * W])
    x = {"tables": torch.where(listed_, order[place], -1).to(torch.int32), "lens": lens.to(torch.int32), "parents": None}
    x["new"] = torch.ones(B, dtype=torch.int32, device="cuda")
    x["held"] = torch.zeros(n_pages, dtype=torch.uint8, device="cuda")
    x["held"][order[-1]] = 1                            # a page that padding writes to
    if W > 1:
        x["parents"] = (req * W + torch.randint(0, W, (B,), generator=g, device="cuda")).to(torch.int32)
    elif case["joins"]:
        p = torch.arange(B, dtype=torch.int32, device="cuda")
        new = torch.randperm(B, generator=g, device="cuda")[:case["joins"]]
        p[new] = -1
        x["new"][new] = torch.randint(1, case["prompt"] + 1, (case["joins"],), generator=g, device="cuda").to(torch.int32)
        x["parents"] = p
    x["max_new"] = B + case["joins"] * case["prompt"]
    return x


def _append_inputs(case, seed):
    g = _gen(seed)
    n, page, c = case["tokens"], case["page"], case["copies"]
    x = {"Kc": _pages(case["pages"], case, g), "Vc": _pages(case["pages"], case, g)}
    shape = (n, case["kv_heads"], case["head_dim"])
    x["K"], x["V"] = (torch.randn(shape, generator=g, device="cuda").to(DTYPES[case["dtype"]]) for _ in range(2))
    order = torch.randperm(case["pages"], generator=g, device="cuda")
    slots = (order[2 * c:, None] * page + torch.arange(page, device="cuda")).flatten()
    first = int(torch.randint(0, page, (1,), generator=g, device="cuda"))
    x["slots"] = slots[first:first + n].clone()
    x["slots"][n - n // 16:] = -1                       # the call is padded to a fixed number of rows
    x["copies"] = None
    if c:
        rows = torch.randint(0, page, (c,), generator=g, device="cuda")
        pair = torch.stack([order[:c], order[c:2 * c], rows], 1)
        x["copies"] = torch.where(rows[:, None] > 0, pair, torch.tensor([-1, -1, 0], device="cuda")).to(torch.int32).contiguous()
    return x


def _select_inputs(case, seed):
    g = _gen(seed)
    B, W, V = case["batch"], case["beams"], case["vocab"]
    x = {"logits": (torch.randn((B, W, V), generator=g, device="cuda") * 3.0).to(DTYPES[case["dtype"]])}
    x["scores"] = -4.0 - 6.0 * torch.rand((B, W), generator=g, device="cuda").sort(dim=1).values
    x["ended"] = torch.zeros((B, W), dtype=torch.uint8, device="cuda")
    if case["ended"]:
        x["ended"] = (torch.rand((B, W), generator=g, device="cuda") < 0.2).to(torch.uint8)
    if case["first"]:                                   # before the first token all beams are the same: one takes part
        x["scores"][:, 1:] = -math.inf
        x["ended"].zero_()
    return x


def prepare(case, seed):
    op = case["op"]
    s = {"attn": _attn_inputs, "step": _step_inputs, "append": _append_inputs, "select": _select_inputs}[op](case, seed)
    s["case"] = case
    B = case.get("batch", 1)
    if op == "step":
        s["out"] = {"tables": torch.full_like(s["tables"], -1), "lens": torch.empty_like(s["lens"]),
                    "cu_new": torch.empty(B + 1, dtype=torch.int32, device="cuda"),
                    "slots": torch.empty(s["max_new"], dtype=torch.int64, device="cuda"),
                    "positions": torch.empty(s["max_new"], dtype=torch.int32, device="cuda"),
                    "copies": torch.empty((B, 3), dtype=torch.int32, device="cuda"),
                    "status": torch.empty(1, dtype=torch.int32, device="cuda")}
    if own:
        from paper_2604_04722_b200 import binding as kq
        s["kq"] = kq
        if op == "attn":
            s["cache"] = kq.kvq_page_cache(s["K"], s["V"])
            s["O"] = torch.empty_like(s["Q"])
            s["lse"] = torch.empty((B, case["q_heads"]), dtype=torch.float32, device="cuda")
            s["bytes"] = kq.kvq_page_attn_workspace_bytes(B, case["q_heads"], case["kv_heads"], case["head_dim"])
            s["work"] = torch.zeros(s["bytes"], dtype=torch.uint8, device="cuda")
        elif op == "append":
            s["cache"] = kq.kvq_page_cache(s["Kc"], s["Vc"])
        elif op == "select":
            shape = (B, case["beams"])
            s["out"] = {"parents": torch.empty(shape, dtype=torch.int32, device="cuda"),
                        "tokens": torch.empty(shape, dtype=torch.int32, device="cuda"),
                        "scores": torch.empty(shape, dtype=torch.float32, device="cuda"),
                        "ended": torch.empty(shape, dtype=torch.uint8, device="cuda")}
    torch.cuda.synchronize()
    return s


# ---------------------------------------------------------------- one pass

END = 2                                                 # the token that ends a sequence


def _plain_attn(s):
    case = s["case"]
    B, H, D, n = case["batch"], case["kv_heads"], case["head_dim"], s["tables"].shape[1] * case["page"]
    at = s["tables"].long().clamp(min=0)
    k = s["K"][at].float().reshape(B, n, H, D).permute(0, 2, 3, 1)
    z = (s["Q"].float().reshape(B, H, -1, D) @ k) * D ** -0.5
    del k
    seen = torch.arange(n, device="cuda") < s["lens"][:, None]
    z = z.masked_fill(~seen[:, None, None, :], -math.inf)
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    total = e.sum(-1, keepdim=True)
    v = s["V"][at].float().reshape(B, n, H, D).masked_fill(~seen[:, :, None, None], 0.0).permute(0, 2, 1, 3)
    o = (e @ v) / torch.where(total == 0, torch.ones_like(total), total)
    return {"O": o.reshape(s["Q"].shape).to(s["Q"].dtype), "lse": (m + torch.log(total)).reshape(B, -1)}


def _plain_step(s):
    case = s["case"]
    B, page, width = case["batch"], case["page"], s["tables"].shape[1]
    dev, n_pages = s["tables"].device, s["held"].numel()
    b, col = torch.arange(B, device=dev), torch.arange(width, device=dev)
    p = b if s["parents"] is None else s["parents"].long()
    old = torch.where(p >= 0, s["lens"].long()[p.clamp(min=0)], 0)
    first = torch.full((B,), B, device=dev).scatter_reduce(0, p.clamp(min=0), torch.where(p >= 0, b, B), "amin")
    copied = (p >= 0) & (old % page > 0) & (first[p.clamp(min=0)] != b)
    kept = torch.where(copied, old // page, (old + page - 1) // page)
    after = old + s["new"].long()
    need = (after + page - 1) // page - kept
    rows = s["tables"][p.clamp(min=0)].long()
    stays, comes = col < kept[:, None], (col >= kept[:, None]) & (col < (kept + need)[:, None])
    used = torch.zeros(n_pages + 1, dtype=torch.bool, device=dev)
    used[torch.where(stays, rows, n_pages)] = True
    free = torch.nonzero(~used[:n_pages] & (s["held"] == 0)).flatten()
    which = (need.cumsum(0) - need)[:, None] + col - kept[:, None]
    tables = torch.where(stays, rows, torch.where(comes, free[which.clamp(0, free.numel() - 1)], s["out"]["tables"].long()))
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), s["new"].long().cumsum(0)])
    t = torch.arange(s["max_new"], device=dev)
    row = torch.searchsorted(cu[1:], t, right=True).clamp(max=B - 1)
    pos = old[row] + t - cu[row]
    there = t < cu[-1]
    slot = tables[row, (pos // page).clamp(max=width - 1)] * page + pos % page
    dst = torch.gather(tables, 1, kept.clamp(max=width - 1)[:, None])[:, 0]
    src = torch.gather(rows, 1, kept.clamp(max=width - 1)[:, None])[:, 0]
    copies = torch.stack([torch.where(copied, src, -1), torch.where(copied, dst, -1), torch.where(copied, old % page, 0)], 1)
    bad = (need.sum() > free.numel()).int() + 2 * (after.max() > width * page).int() + 4 * (cu[-1] > s["max_new"]).int()
    return {"tables": tables.int(), "lens": after.int(), "cu_new": cu.int(), "slots": torch.where(there, slot, -1),
            "positions": torch.where(there, pos, -1).int(), "copies": copies.int(), "status": bad.reshape(1)}


def _plain_append(s):
    page = s["case"]["page"]
    there = torch.nonzero(s["slots"] >= 0).flatten()
    at, off = s["slots"][there] // page, s["slots"][there] % page
    if s["copies"] is not None:
        src, dst, rows = s["copies"].long().unbind(1)
        i = torch.arange(page, device="cuda")
        r, o = torch.nonzero(i < rows[:, None]).unbind(1)
        for c in (s["Kc"], s["Vc"]):
            c[dst[r], o] = c[src[r], o]
    s["Kc"][at, off] = s["K"][there]
    s["Vc"][at, off] = s["V"][there]
    return s["Kc"], s["Vc"]


def _plain_select(s):
    case = s["case"]
    B, W, V = case["batch"], case["beams"], case["vocab"]
    z = s["logits"].double()                            # neighbouring candidates may be closer than 32 bits tell apart
    z = z - z.amax(-1, keepdim=True)
    z = z - torch.log(torch.exp(z).sum(-1, keepdim=True)) + s["scores"].double()[:, :, None]
    ended = s["ended"].bool()
    z = z.masked_fill(ended[:, :, None], -math.inf)
    z[:, :, END] = torch.where(ended, s["scores"].double(), z[:, :, END])
    best, at = torch.sort(z.reshape(B, W * V), dim=1, descending=True, stable=True)
    best, at = best[:, :W], at[:, :W]
    src, tok = at // V, at % V
    there = torch.isfinite(best)
    over = torch.gather(ended, 1, src) | (tok == END) | ~there
    parents = src + torch.arange(B, device="cuda")[:, None] * W
    return {"parents": torch.where(there, parents, -1).int(), "tokens": torch.where(there, tok, -1).int(),
            "scores": torch.where(there, best, -math.inf).float(), "ended": over.to(torch.uint8)}


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"attn": _plain_attn, "step": _plain_step, "append": _plain_append, "select": _plain_select}[op](s)
    kq = s["kq"]
    if op == "attn":
        kq.kvq_page_attn(s["cache"], s["Q"], s["O"], s["lse"], s["tables"], s["tables"].shape[1], s["lens"], case["batch"],
                         case["q_heads"], case["head_dim"] ** -0.5, s["work"], s["bytes"])
        return {"O": s["O"], "lse": s["lse"]}
    if op == "step":
        o = s["out"]
        kq.kvq_page_step(s["tables"], o["tables"], s["tables"].shape[1], s["lens"], o["lens"], s["parents"], s["new"],
                         case["batch"], s["held"], s["held"].numel(), case["page"], s["max_new"], o["cu_new"], o["slots"],
                         o["positions"], o["copies"], o["status"])
        return o
    if op == "append":
        kq.kvq_page_append(s["cache"], s["K"], s["V"], s["slots"], case["tokens"], s["copies"], case["copies"])
        return s["Kc"], s["Vc"]
    o = s["out"]
    dtype = {"fp16": kq.KVQ_FP16, "bf16": kq.KVQ_BF16, "fp32": kq.KVQ_FP32}[case["dtype"]]
    kq.kvq_beam_select(s["logits"], dtype, s["scores"], s["ended"], case["batch"], case["beams"], case["vocab"],
                       case["beams"], END, o["parents"], o["tokens"], o["scores"], o["ended"])
    return o


def work(case):
    """Bytes: cached rows that are seen, queries and outputs once; of a step the listed pages, the page flags and what is
    written; appended rows once in, once out; logits once.  Flops: the two products, one exponential per logit."""
    op = case["op"]
    if op == "attn":
        seen, D, Hq, B = sum(_lens(case)), case["head_dim"], case["q_heads"], case["batch"]
        pages = sum(-(-n // case["page"]) for n in _lens(case))
        return {"bytes": 4 * D * case["kv_heads"] * seen + 4 * pages + B * (4 + Hq * (4 * D + 4)), "flops": 4.0 * D * Hq * seen}
    if op == "step":
        B, n = case["batch"], case["ctx"]
        pages = B * (0.75 * n / case["page"] + 1)       # (rows hold between half of ctx and all of it)
        new = B + case["joins"] * (0.5 * case["prompt"])
        again = 2 if case["beams"] > 1 or case["joins"] else 1
        return {"bytes": 4 * again * pages + case["spare"] + B * 32 + 12 * new, "flops": pages + new}
    if op == "append":
        row = 2 * case["kv_heads"] * case["head_dim"]
        n = case["tokens"] - case["tokens"] // 16
        return {"bytes": 4 * row * (n + case["copies"] * case["page"] / 2) + 8 * case["tokens"], "flops": 0.0}
    size = 4 if case["dtype"] == "fp32" else 2
    read = case["batch"] * case["beams"] * case["vocab"] * (0.8 if case["ended"] else 1.0)
    return {"bytes": size * read + 18 * case["batch"] * case["beams"], "flops": 4.0 * read}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_attn(case, x):
    B, G, D, page = case["batch"], case["q_heads"] // case["kv_heads"], case["head_dim"], case["page"]
    O = torch.zeros(x["Q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(x["Q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lens(case)):
        if n == 0:
            continue
        t = torch.arange(n, device="cuda")
        where = x["tables"][b, t // page].long()
        for h in range(case["kv_heads"]):
            key, value = (c[where, t % page, h].double() for c in (x["K"], x["V"]))
            logit = x["Q"][b, h * G:(h + 1) * G].double() @ key.T / math.sqrt(D)
            top = logit.max(dim=1).values
            weight = torch.exp(logit - top[:, None])
            O[b, h * G:(h + 1) * G] = weight @ value / weight.sum(1)[:, None]
            lse[b, h * G:(h + 1) * G] = top + torch.log(weight.sum(1))
    return {"O": O, "lse": lse}


def _exact_step(case, x):
    """One row after the other, with sets and lists."""
    page, tables, lens = case["page"], x["tables"].tolist(), x["lens"].tolist()
    B, width = len(lens), len(tables[0])
    parents = list(range(B)) if x["parents"] is None else x["parents"].tolist()
    new, held = x["new"].tolist(), x["held"].tolist()
    seen, rows, copies, owned = set(), [], [], set()
    for b, p in enumerate(parents):
        row = tables[p][:-(-lens[p] // page)] if p >= 0 else []
        copies.append([-1, -1, 0])
        if p >= 0 and lens[p] % page and p in seen:
            copies[b] = [row.pop(), None, lens[p] % page]
        if p >= 0:
            seen.add(p)
        owned.update(row)
        rows.append(row)
    free = (i for i in range(len(held)) if not held[i] and i not in owned)
    out = {"lens": [], "cu_new": [0], "slots": [], "positions": [], "status": [0]}
    for b, p in enumerate(parents):
        n = lens[p] if p >= 0 else 0
        while len(rows[b]) * page < n + new[b]:
            rows[b].append(next(free))
        if copies[b][2]:
            copies[b][1] = rows[b][n // page]
        for at in range(n, n + new[b]):
            out["slots"].append(rows[b][at // page] * page + at % page)
            out["positions"].append(at)
        out["lens"].append(n + new[b])
        out["cu_new"].append(out["cu_new"][-1] + new[b])
    for k in ("slots", "positions"):
        out[k] += [-1] * (x["max_new"] - len(out[k]))
    out["tables"], out["copies"] = [r + [-1] * (width - len(r)) for r in rows], copies
    return {k: torch.tensor(out[k], dtype=torch.int64 if k == "slots" else torch.int32)
            for k in ("tables", "lens", "cu_new", "slots", "positions", "copies", "status")}


def _exact_select(case, x):
    W, V = case["beams"], case["vocab"]
    out = {"parents": [], "tokens": [], "scores": [], "ended": []}
    for b in range(case["batch"]):
        pool = []
        for w in range(W):
            score = float(x["scores"][b, w])
            if x["ended"][b, w]:
                pool.append((-score, w, END, 1))
                continue
            z = x["logits"][b, w].double()
            logp = z - torch.logsumexp(z, 0) + score
            kth = torch.topk(logp, min(W, V)).values[-1]
            for v in torch.nonzero(logp >= kth).flatten().tolist():
                pool.append((-float(logp[v]), w, v, int(v == END)))
        pool = sorted(c for c in pool if math.isfinite(c[0]))[:W]
        gone = W - len(pool)
        out["parents"].append([b * W + c[1] for c in pool] + [-1] * gone)
        out["tokens"].append([c[2] for c in pool] + [-1] * gone)
        out["scores"].append([-c[0] for c in pool] + [-math.inf] * gone)
        out["ended"].append([c[3] for c in pool] + [1] * gone)
    kinds = {"parents": torch.int32, "tokens": torch.int32, "scores": torch.float64, "ended": torch.uint8}
    return {k: torch.tensor(out[k], dtype=kinds[k]) for k in kinds}


def exact(case, seed):
    if case["op"] == "attn":
        return _exact_attn(case, _attn_inputs(case, seed))
    if case["op"] == "step":
        return _exact_step(case, _step_inputs(case, seed))
    if case["op"] == "select":
        return _exact_select(case, _select_inputs(case, seed))
    return None                                         # appended rows are moved, not computed
