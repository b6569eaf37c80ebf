"""Cases and plain forms of the operators for speculative decoding and sliding-window layers over the
mixed-precision cache: attention for a tree of drafted tokens, its verification, and windowed decode attention.

Shapes are those of the workloads in ``paper_2604_04722_b200/synth.py`` (SmolLM-135M/360M/1.7B-shaped layers and the
32768-token stress layer).  ``own`` selects between the plain forms below and the framework's entry points.
"""
import math

import torch

own = False

D = 64
MIX = {"cfg1": (0.40, 0.35, 0.20, 0.05), "cfg4": (0.25, 0.40, 0.25, 0.10), "cfg5": (0.50, 0.30, 0.15, 0.05)}
ROW_BYTES = (40, 72, 136, 256)             # packed K + V bytes of one token and KV head, by class


def listed():
    tree = dict(op="tree", ragged=False, chain=False, as_stored=True, window=0, sinks=0)
    win = dict(op="window", ragged=False)
    ver = dict(op="verify", draft=True, chain=False)
    return [
        # a short prompt on the smallest model, a handful of drafted tokens: latency
        dict(tree, name="tree_cfg1_512x8", batch=1, q_heads=9, kv_heads=3, ctx=512, mix="cfg1", nodes=8),
        # one user of the smallest model, a draft model's chain of guesses
        dict(tree, name="tree_cfg2_2048x5_chain", batch=1, q_heads=9, kv_heads=3, ctx=2048, mix="cfg1", nodes=5, chain=True),
        # a batch of grouped-query requests of different lengths, a full tree of 64 nodes each
        dict(tree, name="tree_cfg3_4096x64", batch=8, q_heads=15, kv_heads=5, ctx=4096, mix="cfg1", nodes=64, ragged=True),
        # the same batch in a windowed layer, drafted rows kept in fp16, odd sizes
        dict(tree, name="tree_cfg3_4001x21_w1024", batch=8, q_heads=15, kv_heads=5, ctx=4001, mix="cfg1", nodes=21,
             ragged=True, as_stored=False, window=1024, sinks=4),
        # a large batch on the largest model, and the stress layer: throughput
        dict(tree, name="tree_cfg4_8192x32", batch=16, q_heads=32, kv_heads=32, ctx=8192, mix="cfg4", nodes=32),
        dict(tree, name="tree_cfg5_32768x16", batch=16, q_heads=32, kv_heads=32, ctx=32768, mix="cfg5", nodes=16),
        # one decode step of a windowed layer: one user of a small model, a ragged batch, long contexts
        dict(win, name="window_cfg2_2048_w256", batch=1, q_heads=9, kv_heads=3, ctx=2048, mix="cfg1", window=256, sinks=4),
        dict(win, name="window_cfg3_4096_w1000", batch=8, q_heads=15, kv_heads=5, ctx=4096, mix="cfg1", window=1000,
             sinks=5, ragged=True),
        dict(win, name="window_cfg5_32768_w8192", batch=16, q_heads=32, kv_heads=32, ctx=32768, mix="cfg5", window=8192,
             sinks=4),
        # one user's few guesses; a batch of trees drawn from a draft model; trees of fixed guesses, odd vocabulary
        dict(ver, name="verify_1x8", batch=1, nodes=8, vocab=49152),
        dict(ver, name="verify_16x64", batch=16, nodes=64, vocab=49152),
        dict(ver, name="verify_8x31_guesses", batch=8, nodes=31, vocab=32003, draft=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tree", "tree", "window", "verify"])
    if op == "verify":
        batch, nodes, vocab = _log_int(rng, 1, 32), rng.randint(1, 64), _log_int(rng, 1000, 60000)
        while batch * (nodes + 1) * vocab > 16 * 65 * 49152:
            batch = max(1, batch // 2)
        return dict(op=op, batch=batch, nodes=nodes, vocab=vocab, draft=rng.random() < 0.7, chain=rng.random() < 0.3)
    kv_heads, group = rng.choice([(3, 3), (5, 3), (32, 1), (4, 2), (1, 1), (2, 8)])
    ctx, batch = _log_int(rng, 17, 32768), _log_int(rng, 1, 24)
    while batch * kv_heads * ctx > 8 * 32 * 16384:
        batch, ctx = max(1, batch // 2), ctx if batch > 1 else ctx // 2
    window = _log_int(rng, 1, ctx) if op == "window" or rng.random() < 0.4 else 0
    c = dict(op=op, batch=batch, q_heads=kv_heads * group, kv_heads=kv_heads, ctx=ctx, mix=rng.choice(sorted(MIX)),
             window=window, sinks=rng.randint(0, 8) if window else 0, ragged=rng.random() < 0.5)
    if op == "tree":
        c.update(nodes=rng.randint(1, 64), chain=rng.random() < 0.2, as_stored=rng.random() < 0.7)
        while c["nodes"] * group * batch * kv_heads * ctx > 16 * 16 * 32 * 32768:
            c["nodes"] //= 2
    return c


def _lens(case):
    """Cached tokens per sequence: all ``ctx``, or from about half of it up to ``ctx``."""
    n = case["ctx"]
    return [n - (b * 7919 % (n // 2 + 1) if case["ragged"] else 0) for b in range(case["batch"])]


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows(shape, g):
    """fp16 rows ~ N(0, 1) with four channels per KV head eight times as large (shape [..][kv_heads][64])."""
    x = torch.randn(shape, generator=g, device="cuda")
    H = shape[-2]
    scale = torch.ones(H, D, device="cuda")
    ch = torch.rand(H, D, generator=g, device="cuda").argsort(dim=1)[:, :4]
    scale.scatter_(1, ch, 8.0)
    return (x * scale).half()


def _bits(shape, mix, g):
    u = torch.rand(shape, generator=g, device="cuda")
    edges = torch.tensor(MIX[mix], device="cuda").cumsum(0)[:3]
    return (2 << torch.bucketize(u, edges).to(torch.int32)).to(torch.uint8)


def _parents(batch, nodes, chain, ragged, g):
    """parent of every node: -1 for children of the last cached token, -2 for unused nodes at the end of a row."""
    i = torch.arange(nodes, device="cuda")
    if chain:
        p = (i - 1).expand(batch, nodes).clone()
    else:
        back = torch.randint(1, 6, (batch, nodes), generator=g, device="cuda")
        p = torch.clamp(i - back, min=-1)
    if ragged:
        used = torch.randint(max(1, nodes // 2), nodes + 1, (batch, 1), generator=g, device="cuda")
        p = torch.where(i < used, p, torch.full_like(p, -2))
    return p.to(torch.int32).contiguous()


def _attention_inputs(case, seed):
    g = _gen(seed)
    B, H, n = case["batch"], case["kv_heads"], case["ctx"]
    K, V = _rows((B, n, H, D), g), _rows((B, n, H, D), g)
    x = {"K": K, "V": V, "bits": _bits((B, n), case["mix"], g), "lens": _lens(case)}
    if case["op"] == "tree":
        T = case["nodes"]
        x["Q"] = torch.randn((B, T, case["q_heads"], D), generator=g, device="cuda").half()
        x["Kd"], x["Vd"] = _rows((B, T, H, D), g), _rows((B, T, H, D), g)
        x["bits_d"] = _bits((B, T), case["mix"], g) if case["as_stored"] else None
        x["parents"] = _parents(B, T, case["chain"], case["ragged"], g)
    else:
        x["Q"] = torch.randn((B, case["q_heads"], D), generator=g, device="cuda").half()
    return x


def _verify_inputs(case, seed):
    g = _gen(seed)
    B, T, V = case["batch"], case["nodes"], case["vocab"]
    z = torch.randn((B, T + 1, V), generator=g, device="cuda") * 3.0
    x = {"parents": _parents(B, T, case["chain"], False, g)}
    x["target"] = torch.softmax(z, dim=2)
    q = torch.softmax(z + 0.7 * torch.randn(z.shape, generator=g, device="cuda"), dim=2)
    rows = torch.gather(q, 1, (x["parents"].long() + 1)[:, :, None].expand(B, T, V)).reshape(B * T, V)
    x["tokens"] = torch.multinomial(rows, 1, generator=g).reshape(B, T).to(torch.int32)
    x["draft"] = q if case["draft"] else None
    x["u"] = torch.rand((B, T), generator=g, device="cuda")
    x["u_next"] = torch.rand((B,), generator=g, device="cuda")
    return x


def _quantize(x, bits):
    """The row quantizer: codes, scale and zero-point (all as numbers) of fp16 rows [..][H][64] at bits [..]; 16 keeps
    the row (scale 1, zero-point 0)."""
    f = x.float()
    levels = (2.0 ** bits.float() - 1.0)[..., None, None]
    keep = (bits == 16)[..., None, None]
    lo, hi = f.amin(-1, keepdim=True), f.amax(-1, keepdim=True)
    s = ((hi - lo) / levels).half().float()
    inv = torch.where(s == 0, torch.zeros_like(s), 1.0 / s)
    codes = torch.round(torch.minimum((f - lo) * inv, levels))
    codes = torch.where(keep, f, codes).half()
    return codes, torch.where(keep, torch.ones_like(s), s), torch.where(keep, torch.zeros_like(lo), lo)


class _Handle:
    """A cache handle that is freed with the state that holds it."""

    def __init__(self, kq, case, x):
        mix = MIX[case["mix"]]
        B, H, n = case["batch"], case["kv_heads"], case["ctx"]
        mean = sum(p * r for p, r in zip(mix, ROW_BYTES))
        budget = int(1.2 * mean * B * H * n) + (4 * B * H + 8) * 2 * 65536
        self.kq, self.ctx = kq, kq.kvq_create_arena(1, case["q_heads"], H, D, n, B, budget)
        if case["ragged"]:
            kq.kvq_append_ragged(self.ctx, 0, x["K"], x["V"], x["bits"], None, n, x["lens"])
        else:
            kq.kvq_append(self.ctx, 0, x["K"], x["V"], x["bits"], n)

    def __del__(self):
        self.kq.kvq_destroy(self.ctx)


def prepare(case, seed):
    if case["op"] == "verify":
        s = dict(_verify_inputs(case, seed), case=case)
        if own:
            from paper_2604_04722_b200 import binding
            B, T = case["batch"], case["nodes"]
            s["kq"] = binding
            s["n_accepted"] = torch.empty(B, dtype=torch.int32, device="cuda")
            s["path"] = torch.empty((B, T), dtype=torch.int32, device="cuda")
            s["next"] = torch.empty(B, dtype=torch.int32, device="cuda")
        return s
    x = _attention_inputs(case, seed)
    s = {k: v for k, v in x.items() if k not in ("K", "V", "bits")}
    s["case"] = case
    if own:                                            # the cache is a handle of the library, filled by its append
        from paper_2604_04722_b200 import binding
        s["kq"], s["handle"] = binding, _Handle(binding, case, x)
        s["O"] = torch.empty_like(x["Q"])
    else:                                              # the cache is what was stored: codes, scales, zero-points
        parts = [(_quantize(x["K"][b], x["bits"][b]), _quantize(x["V"][b], x["bits"][b])) for b in range(case["batch"])]
        for name, w in (("K", 0), ("V", 1)):
            s[name] = tuple(torch.stack([p[w][k] for p in parts]) for k in range(3))
        s["n"] = torch.tensor(x["lens"], device="cuda")
    torch.cuda.synchronize()
    return s


# ---------------------------------------------------------------- one pass

def _values(stored):
    codes, scale, zero = stored
    return codes.float() * scale + zero


def _softmax_rows(z):
    """Softmax over the last axis; a row that sees nothing has weights zero."""
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, torch.ones_like(total), total)


def _attend(q, k, v, seen):
    """q [B][T][Hq][64], k, v [B][n][H][64], seen [B][T][n] -> [B][T][Hq][64], all in 32 bits."""
    B, T, Hq, _ = q.shape
    H = k.shape[2]
    qh = q.float().reshape(B, T, H, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)
    z = (qh @ k.permute(0, 2, 3, 1)) * 0.125
    z = z.reshape(B, H, T, Hq // H, -1).masked_fill(~seen[:, None, :, None, :], -math.inf)
    o = _softmax_rows(z).reshape(B, H, T * (Hq // H), -1) @ v.permute(0, 2, 1, 3)
    return o.reshape(B, H, T, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D)


def _plain_tree(s):
    case = s["case"]
    T, n, par = case["nodes"], case["ctx"], s["parents"].long()
    dev = par.device
    i = torch.arange(T, device=dev)
    ok = (par >= -1) & (par < i)
    # ancestors (a node is its own): the chain of parents, doubled until it covers any depth
    step = torch.nn.functional.one_hot(torch.where(ok, par, torch.full_like(par, -1)) + 1, T + 1)[..., 1:].float()
    anc = torch.eye(T, device=dev) + step
    hop = step
    for _ in range(6):
        hop = hop @ hop
        anc = anc + hop @ anc
    anc = anc > 0
    used = ok & ~(anc & ~ok[:, None, :]).any(-1)
    depth = anc.sum(-1) - 1
    pos = s["n"][:, None] + depth
    at = torch.cat([torch.arange(n, device=dev).expand(len(s["n"]), n), pos], dim=1)
    seen = torch.cat([(at[:, :n] < s["n"][:, None])[:, None, :].expand(-1, T, -1), anc], dim=2) & used[:, :, None]
    if case["window"]:
        seen = seen & ((at[:, None, :] > pos[:, :, None] - case["window"]) | (at[:, None, :] < case["sinks"]))
    if s["bits_d"] is None:
        kd, vd = s["Kd"].float(), s["Vd"].float()
    else:
        kd, vd = _values(_quantize(s["Kd"], s["bits_d"])), _values(_quantize(s["Vd"], s["bits_d"]))
    return _attend(s["Q"], torch.cat([_values(s["K"]), kd], 1), torch.cat([_values(s["V"]), vd], 1), seen).half()


def _plain_window(s):
    case = s["case"]
    at, n = torch.arange(case["ctx"], device="cuda"), s["n"][:, None]
    seen = (at < n) & ((at >= n - case["window"]) | (at < case["sinks"]))
    return _attend(s["Q"][:, None], _values(s["K"]), _values(s["V"]), seen[:, None])[:, 0].half()


def _plain_verify(s):
    case, par, tok = s["case"], s["parents"].long() + 1, s["tokens"].long()
    B, T, V = case["batch"], case["nodes"], case["vocab"]
    b = torch.arange(B, device="cuda")
    cur, c, Z = torch.zeros_like(b), torch.zeros(B, device="cuda").double(), torch.ones(B, device="cuda").double()
    gone = torch.zeros((B, V), dtype=torch.bool, device="cuda")        # fixed guesses that were turned down
    path, count = torch.full((B, T), -1, dtype=torch.int32, device="cuda"), torch.zeros_like(b)

    def residual():
        p = s["target"][b, cur].double()
        return p.masked_fill(gone, 0.0) if s["draft"] is None else torch.clamp(p - c[:, None] * s["draft"][b, cur].double(), min=0.0)

    for i in range(T):                                 # a child comes after its parent: one walk in index order
        tested = par[:, i] == cur
        r = residual()
        q = 1.0 if s["draft"] is None else s["draft"][b, cur, tok[:, i]].double()
        took = tested & (s["u"][:, i].double() * Z * q < r[b, tok[:, i]])
        lost = tested & ~took
        path[b, count] = torch.where(took, torch.full_like(cur, i).int(), path[b, count.clamp(max=T - 1)])
        count = count + took
        cur = torch.where(took, torch.full_like(cur, i + 1), cur)
        if s["draft"] is None:
            Z = torch.where(lost, Z - r[b, tok[:, i]], Z)
            gone[b, tok[:, i]] = gone[b, tok[:, i]] | lost
            gone = gone & ~took[:, None]
            Z = torch.where(took, torch.ones_like(Z), Z)
        else:
            c = torch.where(lost, c + Z, torch.where(took, torch.zeros_like(c), c))
            Z = torch.where(lost, residual().sum(1), torch.where(took, torch.ones_like(Z), Z))
    r = residual()
    r = torch.where(r.sum(1, keepdim=True) > 0, r, s["target"][b, cur].double())
    run = r.cumsum(1)
    token = (run <= s["u_next"].double()[:, None] * run[:, -1:]).sum(1)
    return {"n_accepted": count.int(), "path": path, "next": token.clamp(max=V - 1).int()}


def run(s):
    case = s["case"]
    if not own:
        return {"tree": _plain_tree, "window": _plain_window, "verify": _plain_verify}[case["op"]](s)
    kq = s["kq"]
    if case["op"] == "tree":
        kq.kvq_attend_tree(s["handle"].ctx, 0, s["Q"], s["Kd"], s["Vd"], s["bits_d"], s["parents"], case["nodes"], s["O"],
                           case["window"], case["sinks"])
        return s["O"]
    if case["op"] == "window":
        kq.kvq_decode_attn_window(s["handle"].ctx, 0, s["Q"], s["O"], case["window"], case["sinks"])
        return s["O"]
    kq.kvq_verify_tree(s["target"], s["draft"], s["tokens"], s["parents"], case["batch"], case["nodes"], case["vocab"],
                       s["u"], s["u_next"], s["n_accepted"], s["path"], s["next"])
    return {"n_accepted": s["n_accepted"], "path": s["path"], "next": s["next"]}


def work(case):
    """Bytes: every visible cached row once, queries, drafted rows and outputs once; for the verification the final
    rows of both distributions (which rows are read before depends on the draws).  Flops: the two products."""
    B, T = case["batch"], case.get("nodes", 1)
    if case["op"] == "verify":
        return {"bytes": B * (4 * case["vocab"] * (2 if case["draft"] else 1) + T * 20 + 12), "flops": 2.0 * B * case["vocab"]}
    H, Hq = case["kv_heads"], case["q_heads"]
    row = sum(p * r for p, r in zip(MIX[case["mix"]], ROW_BYTES))
    seen = sum(min(n, case["window"] + case["sinks"]) if case["window"] else n for n in _lens(case))
    bytes_ = seen * H * row + 2 * 2 * D * B * T * Hq
    if case["op"] == "tree":
        bytes_ += B * T * (4 * D * H + 5)
    return {"bytes": bytes_, "flops": 4.0 * D * T * Hq * seen}


# ---------------------------------------------------------------- the definitions in 64 bits

def _stored64(x, bits):
    """What a row of fp16 values [H][64] is worth after being stored with the given number of bits."""
    if bits == 16:
        return x.double()
    lo = x.min(dim=-1, keepdim=True).values.float()
    span = x.max(dim=-1, keepdim=True).values.float() - lo
    scale = span.div(2 ** bits - 1).half().float()
    code = torch.where(scale > 0, x.float().sub(lo).mul(scale.reciprocal()), torch.zeros_like(x.float()))
    return code.clamp(max=2 ** bits - 1).round().double() * scale.double() + lo.double()


def _stored_rows64(x, bits):
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for b in (2, 4, 8, 16):
        at = (bits == b).nonzero().flatten()
        if at.numel():
            out[at] = _stored64(x[at], b)
    return out


def _exact_verify(case, x):
    out = {"n_accepted": [], "path": [], "next": []}
    parents, tokens = x["parents"].tolist(), x["tokens"].tolist()
    for b in range(case["batch"]):
        at, path = -1, []
        while True:                                    # at every accepted node its children are asked in turn
            left = x["target"][b, at + 1].double()
            mass, q = 1.0, None if x["draft"] is None else x["draft"][b, at + 1].double()
            found = None
            for i in [j for j in range(case["nodes"]) if parents[b][j] == at]:
                t = tokens[b][i]
                if x["u"][b, i].double() * mass * (1.0 if q is None else q[t]) < left[t]:
                    found = i
                    break
                if q is None:
                    mass = mass - float(left[t])
                    left = left.clone()
                    left[t] = 0.0
                else:
                    left = (left - mass * q).clamp(min=0.0)
                    mass = float(left.sum())
            if found is None:
                break
            path.append(found)
            at = found
        if float(left.sum()) <= 0.0:
            left = x["target"][b, at + 1].double()
        sums = left.cumsum(0)
        out["n_accepted"].append(len(path))
        out["path"].append(path + [-1] * (case["nodes"] - len(path)))
        out["next"].append(int((sums > x["u_next"][b].double() * sums[-1]).nonzero()[0]))
    return {k: torch.tensor(v, dtype=torch.int32) for k, v in out.items()}


def exact(case, seed):
    if case["op"] == "verify":
        return _exact_verify(case, _verify_inputs(case, seed))
    x = _attention_inputs(case, seed)
    B, Hq, group = case["batch"], case["q_heads"], case["q_heads"] // case["kv_heads"]
    Q = x["Q"] if case["op"] == "tree" else x["Q"][:, None]
    out = torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
    for b in range(B):
        n = x["lens"][b]
        k, v = _stored_rows64(x["K"][b, :n], x["bits"][b, :n]), _stored_rows64(x["V"][b, :n], x["bits"][b, :n])
        place = list(range(n))
        if case["op"] == "tree":
            full = torch.full((case["nodes"],), 16, device="cuda") if x["bits_d"] is None else x["bits_d"][b]
            k, v = (torch.cat([c, _stored_rows64(d, full)]) for c, d in ((k, x["Kd"][b]), (v, x["Vd"][b])))
            par = x["parents"][b].tolist()
            chains, use = [], []
            for i, p in enumerate(par):                # the nodes from this one up to its root
                fine = -1 <= p < i and (p < 0 or use[p])
                use.append(fine)
                chains.append([i] + (chains[p] if fine and p >= 0 else []))
            place += [n + len(c) - 1 for c in chains]
            mine, own_place = chains, place[n:]
        else:
            mine, own_place, use = [[]], [n - 1], [True]
        place = torch.tensor(place, device="cuda")
        sight = torch.zeros((len(mine), place.numel()), dtype=torch.bool, device="cuda")
        sight[:, :n] = True
        for i, c in enumerate(mine):
            sight[i, torch.tensor([n + a for a in c], dtype=torch.long, device="cuda")] = True
        if case["window"]:
            near = torch.tensor(own_place, device="cuda")[:, None] - place[None, :] < case["window"]
            sight &= near | (place < case["sinks"])
        sight &= torch.tensor(use, device="cuda")[:, None]
        for h in range(Hq):
            kh, vh = k[:, h // group], v[:, h // group]
            logit = torch.where(sight, Q[b, :, h].double() @ kh.T / math.sqrt(D), torch.tensor(-math.inf, device="cuda").double())
            top = logit.max(1, keepdim=True).values
            w = torch.exp(logit - torch.where(top == -math.inf, torch.zeros_like(top), top))
            out[b, :, h] = (w @ vh) / w.sum(1, keepdim=True).clamp(min=1e-300)
    return out if case["op"] == "tree" else out[:, 0]
