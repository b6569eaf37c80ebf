"""64-bit references of the many-row attention (drafted trees, windows) and of the draft verification, written from
their definitions, with the error bounds the fp16 kernels are held to."""
from __future__ import annotations

import math

import numpy as np

HALF_STEP = 2.0 ** -11          # fp16: a rounding is off by at most this, relative to the value


def dequantize(oracle, codes, meta, bits):
    """Canonical rows [n][H][128] u8, meta [n][H][2] u16, bits [n] -> (code * scale, zero-point) in fp64: the value of an
    element is their sum.  16-bit rows have the value in the first and zero in the second."""
    n, H = codes.shape[:2]
    cs, z = np.zeros((n, H, 64)), np.zeros((n, H, 1))
    m = meta.view(np.float16).astype(np.float64)
    for b in (2, 4, 8):
        at = np.flatnonzero(bits == b)
        if at.size:
            cs[at] = oracle._unpack_codes(codes[at], 64, b).astype(np.float64) * m[at][..., :1]
            z[at] = m[at][..., 1:]
    at = np.flatnonzero(bits == 16)
    if at.size:
        cs[at] = np.ascontiguousarray(codes[at]).view(np.float16).astype(np.float64)
    return cs, z


def quantized(oracle, X, bits):
    """The same for fp16 rows [n][H][64] that are stored at ``bits``."""
    codes, meta, _, _ = oracle.append(X[None], X[None], bits[None])
    return dequantize(oracle, codes[0], meta[0], bits)


def chains(parents):
    """Per node the list [itself, parent, ...] up to its root, or None for a node that is not in use."""
    out = []
    for i, p in enumerate(int(x) for x in parents):
        if p < -1 or p >= i or (p >= 0 and out[p] is None):
            out.append(None)
        else:
            out.append([i] + (out[p] if p >= 0 else []))
    return out


def attention(oracle, cache, lens, Q, group, window=0, sinks=0, tree=None):
    """cache: OracleCache; Q fp16 [B][T][Hq][64]; tree: None (one row, the last cached token's) or a tuple
    (K, V, bits or None, parents).  Returns (O fp64, bound) of Q's shape: what a kernel that rounds each V weight and
    the output to fp16, drafted rows too, and accumulates in fp32 may be off by."""
    B, T, Hq, D = Q.shape
    out, bound = np.zeros(Q.shape), np.zeros(Q.shape)
    for b in range(B):
        n = int(lens[b])
        kcs, kz = dequantize(oracle, cache.kc[b, :n], cache.km[b, :n], cache.bits[b, :n])
        vcs, vz = dequantize(oracle, cache.vc[b, :n], cache.vm[b, :n], cache.bits[b, :n])
        place = list(range(n))
        if tree is None:
            rows = [(0, n - 1, [])] if n else []
        else:
            K, V, bits, parents = tree
            db = np.full(T, 16, np.uint8) if bits is None else bits[b]
            with np.errstate(invalid="ignore"):
                dk, dkz = quantized(oracle, K[b], db)
                dv, dvz = quantized(oracle, V[b], db)
            ch = chains(parents[b])
            place += [n + (len(c) - 1 if c else 0) for c in ch]
            rows = [(i, n + len(c) - 1, [n + a for a in c]) for i, c in enumerate(ch) if c]
            for a, z in ((dk, dkz), (dv, dvz)):        # a drafted row is put together (and rounded) before it is used
                a += z
                z[:] = 0.0
            kcs, kz = np.concatenate([kcs, dk]), np.concatenate([kz, dkz])
            vcs, vz = np.concatenate([vcs, dv]), np.concatenate([vz, dvz])
        place = np.array(place)
        drafted = np.arange(place.size) >= n
        for i, pos, mine in rows:
            see = np.zeros(place.size, bool)
            see[:n] = True
            see[mine] = True
            if window:
                see &= (pos - place < window) | (place < sinks)
            at = np.flatnonzero(see)
            if not at.size:
                continue
            for h in range(Hq):
                q = Q[b, i, h].astype(np.float64)
                kc_, kz_, vc_, vz_ = kcs[at, h // group], kz[at, h // group], vcs[at, h // group], vz[at, h // group]
                logit = (kc_ + kz_) @ q / math.sqrt(D)
                p = np.exp(logit - logit.max())
                p /= p.sum()
                out[b, i, h] = p @ (vc_ + vz_)
                # logits: 64 products of exact factors and a few operations summed in fp32 (a matrix instruction may
                # truncate: 2^-22 per addition, of the running absolute sum); drafted keys are rounded to fp16
                size = (np.abs(kc_) @ np.abs(q) + np.abs(kz_[:, 0]) * abs(q).sum()) / math.sqrt(D)
                off = 80 * 2.0 ** -22 * size + np.where(drafted[at], HALF_STEP * size, 0.0) + 2.0 ** -20
                # a weight's relative error counts twice (its own and the normaliser's); fp16 weights once more;
                # drafted values once more
                rel = np.expm1(off + off.max()) + HALF_STEP + np.where(drafted[at], HALF_STEP, 0.0) + 2.0 ** -18
                spread = (p * rel) @ (np.abs(vc_) + np.abs(vz_))
                bound[b, i, h] = spread + HALF_STEP * (np.abs(out[b, i, h]) + spread) + 2.0 ** -24
    return out, bound


def verify(target, draft, tokens, parents, u, u_next):
    """(path, next token) of one sequence: the children of the node reached so far are asked in turn; a rejection
    replaces the target by the normalised residual.  The residual is kept explicitly here."""
    at, path = -1, []
    while True:
        left, mass = target[at + 1].astype(np.float64), 1.0
        q = None if draft is None else draft[at + 1].astype(np.float64)
        found = None
        for i in (j for j in range(len(tokens)) if parents[j] == at and -1 <= parents[j] < j):
            t = int(tokens[i])
            known = 0 <= t < left.size
            if known and float(u[i]) * mass * (1.0 if q is None else q[t]) < left[t]:
                found = i
                break
            if q is None:
                if known:
                    mass -= left[t]
                    left[t] = 0.0
            else:
                left = np.maximum(left - mass * q, 0.0)
                mass = left.sum()
        if found is None:
            break
        path.append(found)
        at = found
    if not left.sum() > 0:
        left = target[at + 1].astype(np.float64)
    if not left.sum() > 0:
        return path, -1
    run = np.cumsum(left)
    over = np.flatnonzero((run > float(u_next) * run[-1]) & (left > 0))
    return path, int(over[0]) if over.size else int(np.flatnonzero(left > 0)[-1])
