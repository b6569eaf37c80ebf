"""Seeded random calls of the paged cache and of the selection against the definitions in 64 bits: KVQ_RANDOM_CASES sets how many of each
(GPU)."""
import math
import os

import numpy as np
import pytest

import pages_reference as pr
import test_gpu_beams as beams
import test_gpu_pages as pages

pytestmark = pytest.mark.gpu

CASES = int(os.environ.get("KVQ_RANDOM_CASES", "8"))     # more seeds for a longer soak
FIRST = 10000                                          # (the other files' seeds lie below)


@pytest.fixture(scope="module")
def kq():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_04722_b200 import binding, build
    build.build()
    torch.cuda.set_device(0)
    return binding


@pytest.mark.parametrize("seed", range(FIRST, FIRST + CASES))
def test_step(kq, seed):
    rng = np.random.default_rng(seed)
    B, page = int(np.exp(rng.uniform(0, np.log(1500)))), int(rng.choice([1, 2, 8, 16, 31, 64]))
    longest = int(rng.integers(0, 30 * page))
    width, n_pages = longest // page + 3, int(B * (longest / page + 1) * rng.choice([1.01, 1.3]) + 4)
    groups, mode = int(rng.choice([1, 2, 4])), rng.integers(4)
    _, tables, lens = pages._state(seed, B, page, longest, n_pages, width, groups)
    parents = [None, rng.integers(-1, B, B), np.minimum(np.arange(B) // groups * groups + rng.integers(0, groups, B), B - 1),
               np.where(rng.random(B) < 0.3, -1, np.arange(B))][mode]
    new = rng.integers(0, int(rng.choice([2, page + 1, 3 * page])), B)
    max_new = int(new.sum() * rng.choice([0.9, 1, 1.5])) + 1
    held = (rng.random(n_pages) < 0.02).astype(np.uint8) if rng.random() < 0.5 else None
    in_place = bool(mode == 0 and rng.random() < 0.5)
    got = pages.Step(kq, tables, lens, parents, new, held, n_pages, page, max_new, in_place).run()
    want = pr.step(tables, lens, parents, new, held, n_pages, page, max_new)
    pages._check_step(got, tables if in_place else np.full(tables.shape, -77), want, lens)
    if want is None:
        pages._unchanged(got, tables, lens, page)


@pytest.mark.parametrize("seed", range(FIRST, FIRST + CASES))
def test_attention(kq, seed):
    import torch
    rng = np.random.default_rng(seed)
    kv, group = int(rng.choice([1, 1, 2, 3, 4, 5, 8, 12, 32])), int(rng.choice([1, 1, 2, 3, 4, 7, 8, 9, 12, 16, 17, 33]))
    D, page = int(rng.choice([64, 64, 128])), int(rng.choice([1, 5, 8, 16, 16, 24, 64, 200]))
    rows, top = int(np.exp(rng.uniform(0, np.log(300)))), int(np.exp(rng.uniform(0, np.log(20000))))
    while rows * kv * top * D > 3e8:
        rows, top = max(1, rows // 2), top if rows > 1 else top // 2
    lens = [rng.integers(0, top + 1, rows), np.full(rows, top), np.where(rng.random(rows) < 0.1, top, rng.integers(0, max(2, top // 20), rows))][rng.integers(3)]
    a = pages.Attn(kq, lens, kv * group, kv, D, page, str(rng.choice(["fp16", "bf16"])), str(rng.choice(["slots", "heads", "together"])), seed=seed,
                   sharp=float(rng.choice([1, 1, 4])), width=max(1, -(-int(max(lens)) // page)) * int(rng.choice([1, 1, 4])), bad=float(rng.choice([0, 0, 0, 0.1])))
    for _ in range(2):
        a.call()
    torch.cuda.synchronize()
    O, lse, Q = (x.double().cpu().numpy() for x in (a.O, a.lse, a.Q))
    assert np.isfinite(O).all() and not a.work[:4096].any()
    for b in {*rng.integers(0, rows, 6).tolist(), 0, rows - 1, int(np.argmax(lens))}:
        h = int(rng.integers(kv))
        at, (k, v) = slice(h * group, h * group + group), (x[a.live[b]][:, h] for x in a.rows[b])
        o, l, err, lerr = pr.attend(Q[b, at], k, v, a.scale, a.mantissa)
        assert np.all(np.abs(O[b, at] - o) <= err), (b, h)
        assert np.all(np.abs(lse[b, at] - l) <= lerr) if len(k) else np.all(lse[b, at] == -math.inf)


@pytest.mark.parametrize("seed", range(FIRST, FIRST + CASES))
def test_selection(kq, seed):
    """The best candidates, in order up to those that are closer than the sums of exponentials are good to."""
    import torch
    rng = np.random.default_rng(seed)
    B, W, V = int(np.exp(rng.uniform(0, np.log(120)))), int(rng.integers(1, 33)), int(np.exp(rng.uniform(0, np.log(60000))))
    while B * W * V > 6e6:
        B, V = max(1, B // 2), V if B > 1 else V // 2
    n = int(rng.choice([W, W, rng.integers(1, 33)]))
    z = beams._logits(seed, B, W, V, beams._dtypes()[rng.integers(3)], float(rng.choice([0.01, 1, 3, 10])))
    if rng.random() < 0.2:
        z = z.round()
    if rng.random() < 0.2:
        z[torch.rand(z.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") < 0.5] = -math.inf
    s = -rng.uniform(0, float(rng.choice([0.1, 3, 30])), (B, W)).astype(np.float32)
    if rng.random() < 0.2:
        s[:, 1:] = -np.inf
    end = int(rng.integers(-1, V))
    finished = (rng.random((B, W)) < rng.choice([0.2, 0.9])).astype(np.uint8) if end >= 0 and rng.random() < 0.5 else np.zeros((B, W), np.uint8)
    parents, tokens, out, over = beams._run(kq, z, s, finished if end >= 0 else None, n, end)
    x = z.double().cpu().numpy()
    for b in range(B):
        want = pr.select(x[b], s[b], finished[b], n, end)
        k = len(want)
        assert np.all(parents[b, k:] == -1) and np.all(tokens[b, k:] == -1) and np.all(out[b, k:] == -math.inf) and np.all(over[b, k:] == 1)
        w, t = parents[b, :k] - b * W, tokens[b, :k]
        assert np.all((w >= 0) & (w < W)) and len(set(zip(w.tolist(), t.tolist()))) == k
        top = x[b].max(1)
        score = [float(s[b, i]) if finished[b, i] else float(s[b, i]) + x[b, i, j] - top[i] - math.log(np.exp(x[b, i] - top[i]).sum()) for i, j in zip(w, t)]
        best = np.array([c[0] for c in want])
        assert np.all(np.abs(np.array(score) - best) <= 2.0 ** -20) and np.all(np.abs(out[b, :k] - best) <= 2.0 ** -20 + 2.0 ** -24 * np.abs(best))
        assert over[b, :k].tolist() == [int(finished[b, i] != 0 or j == end) for i, j in zip(w, t)]
