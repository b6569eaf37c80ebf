"""The paged cache and beam search in 64 bits: plain definitions, one row after the other."""
import math

import numpy as np


def step(tables, lens, parents, new_lens, held, n_pages, page_size, max_new):
    """One step of the block tables; returns None for a step that does not take place."""
    B, width = tables.shape
    parents = list(range(B)) if parents is None else [int(p) for p in parents]
    rows, copies, seen = [], [], set()
    for p in parents:
        if not -1 <= p < B or (p >= 0 and not 0 <= lens[p] <= width * page_size):
            return None
        row = [int(x) for x in tables[p, :-(-int(lens[p]) // page_size)]] if p >= 0 else []
        if any(not 0 <= x < n_pages for x in row):
            return None
        copy = [-1, -1, 0]
        if p >= 0 and lens[p] % page_size and p in seen:
            copy = [row.pop(), None, int(lens[p]) % page_size]
        seen.add(p)
        rows.append(row)
        copies.append(copy)
    used = {x for row in rows for x in row}
    free = [x for x in range(n_pages) if x not in used and not (held is not None and held[x])]
    out_lens, cu, slots, positions, taken = [], [0], [], [], 0
    for b, p in enumerate(parents):
        n, m = (int(lens[p]) if p >= 0 else 0), int(new_lens[b])
        if m < 0 or n + m > width * page_size:
            return None
        while len(rows[b]) * page_size < n + m:
            if taken == len(free):
                return None
            rows[b].append(free[taken])
            taken += 1
        if copies[b][2]:
            copies[b][1] = rows[b][n // page_size]
        for at in range(n, n + m):
            slots.append(rows[b][at // page_size] * page_size + at % page_size)
            positions.append(at)
        out_lens.append(n + m)
        cu.append(cu[-1] + m)
    if len(slots) > max_new:
        return None
    pad = [-1] * (max_new - len(slots))
    return dict(rows=rows, lens=out_lens, cu_new=cu, slots=slots + pad, positions=positions + pad, copies=copies)


def attend(q, k, v, scale, mantissa):
    """q [G][D], k, v [n][D] (fp64 arrays of the stored values): output, log-sum-exp, and how far the kernel may be from both.

    The kernel's errors: a logit is an fp32 sum of D exact products that the matrix instruction adds 16 at a time, each
    sum cut to 22 bits at worst, and two roundings of the scaled logit; the exponential is good to 2^-22; a weight is held by two 16-bit
    numbers (relative 2^-2p for p bits; fp16 besides not below 2^-25 of the largest weight); n / 16 cut additions; one rounding to the output's type.
    """
    p = mantissa                                       # 11: fp16, 8: bf16 (half a step is 2^-p of the value)
    n, D = k.shape
    if n == 0:
        return np.zeros_like(q), np.full(len(q), -math.inf), np.zeros_like(q), np.zeros(len(q))
    z = (q @ k.T) * scale
    top = z.max(1, keepdims=True)
    w = np.exp(z - top)
    total = w.sum(1, keepdims=True)
    o = (w @ v) / total
    lse = (top + np.log(total))[:, 0]
    logit = ((D / 16 + 2) * 2.0 ** -22 * abs(scale) * (np.abs(q) @ np.abs(k).T) + 2.0 ** -22 * np.abs(z - top) + 2.0 ** -22 * np.abs(z)).max(1, keepdims=True)
    sums = (n / 16 + 64) * 2.0 ** -22
    around = (w @ np.abs(v)) / total
    err = (2 * logit + 2.0 ** -21 + 2.0 ** (-2 * p) + sums) * around + 2.0 ** -p * np.abs(o) + 2.0 ** -25
    if p == 11:
        err = err + 2.0 ** -25 * np.abs(v).sum(0) / total
    return o, lse, err, logit[:, 0] + sums + 2.0 ** -22 * (1 + np.abs(lse))


def select(logits, scores, finished, n_out, end_token):
    """One request: logits [W][V], scores [W], finished [W]; candidates (score, beam, token, ended), best first."""
    pool = []
    for w in range(len(scores)):
        s = float(scores[w])
        if not math.isfinite(s):
            continue
        if finished[w]:
            pool.append((-s, w, end_token, 1))
            continue
        z = logits[w].astype(np.float64)
        top = z.max()
        if not math.isfinite(top) or np.isnan(z).any():
            continue
        logp = s + ((z - top) - math.log(np.exp(z - top).sum()))
        best = np.argsort(-logp, kind="stable")[:n_out]
        pool += [(-float(logp[t]), w, int(t), int(t == end_token)) for t in best if math.isfinite(logp[t])]
    return [(-c[0], *c[1:]) for c in sorted(pool)[:n_out]]
