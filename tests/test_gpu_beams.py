"""The selection of beams against its definition in 64 bits (GPU): beams and tokens have to agree, scores to a few roundings."""
import math

import numpy as np
import pytest

import pages_reference as pr

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kq():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_04722_b200 import binding, build
    build.build()
    torch.cuda.set_device(0)
    return binding


def _run(kq, logits, scores, finished, n_out, end):
    """logits: a CUDA tensor [B][W][V] (a contiguous view is fine)."""
    import torch
    B, W, V = logits.shape
    dtype = {torch.float16: kq.KVQ_FP16, torch.bfloat16: kq.KVQ_BF16, torch.float32: kq.KVQ_FP32}[logits.dtype]
    i32 = lambda: torch.full((B, n_out), -77, dtype=torch.int32, device="cuda")
    parents, tokens, over = i32(), i32(), torch.full((B, n_out), 77, dtype=torch.uint8, device="cuda")
    out = torch.full((B, n_out), float("nan"), device="cuda")
    s = torch.tensor(np.asarray(scores), dtype=torch.float32).cuda()
    f = None if finished is None else torch.tensor(np.asarray(finished), dtype=torch.uint8).cuda()
    kq.kvq_beam_select(logits, dtype, s, f, B, W, V, n_out, end, parents, tokens, out, over)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in (parents, tokens, out, over)]


def _check(kq, logits, scores, finished, n_out, end):
    got = _run(kq, logits, scores, finished, n_out, end)
    parents, tokens, out, over = got
    z = logits.float().cpu().numpy()
    B, W, V = z.shape
    for b in range(B):
        want = pr.select(z[b], scores[b], [0] * W if finished is None else finished[b], n_out, end)
        k = len(want)
        assert parents[b, :k].tolist() == [b * W + c[1] for c in want], b
        assert tokens[b, :k].tolist() == [c[2] for c in want], b
        assert over[b, :k].tolist() == [c[3] for c in want], b
        # the sum of exponentials: fp32 within 16 entries, 2^-21 relative in all; then one rounding to fp32
        assert np.all(np.abs(out[b, :k] - [c[0] for c in want]) <= 2.0 ** -20 + 2.0 ** -24 * np.abs([c[0] for c in want])), b
        assert np.all(parents[b, k:] == -1) and np.all(tokens[b, k:] == -1) and np.all(out[b, k:] == -math.inf) and np.all(over[b, k:] == 1)
    return got


def _logits(seed, B, W, V, dtype, spread=3.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((B, W, V), generator=g, device="cuda") * spread).to(dtype)


def _scores(seed, B, W):
    return -np.random.default_rng(seed).uniform(1, 12, (B, W)).astype(np.float32)


def _dtypes():
    import torch
    return [torch.float16, torch.bfloat16, torch.float32]


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("V", [1, 2, 31, 511, 513, 4099, 32003, 50000])
@pytest.mark.parametrize("B,W,n", [(1, 1, 1), (1, 4, 4), (3, 5, 5), (2, 32, 32), (5, 3, 32), (2, 17, 1)])
def test_selection(kq, B, W, n, V, kind):
    dtype = _dtypes()[kind]
    _check(kq, _logits(V + W, B, W, V, dtype), _scores(V, B, W), None, n, -1)


@pytest.mark.parametrize("seed", range(40))
def test_selection_of_any_shape(kq, seed):
    """Any shape, spread of logits and scores (one beam may hold all of the best), masks, ended beams, first steps, rounded logits with ties."""
    import torch
    rng = np.random.default_rng(seed)
    B, W, V = int(np.exp(rng.uniform(0, np.log(120)))), int(rng.integers(1, 33)), int(np.exp(rng.uniform(0, np.log(60000))))
    while B * W * V > 3e6:
        B, V = max(1, B // 2), V if B > 1 else V // 2
    z = _logits(seed, B, W, V, _dtypes()[rng.integers(3)], float(rng.choice([0.01, 1, 3, 10])))
    if rng.random() < 0.2:
        z = z.round()
    if rng.random() < 0.2:
        z[torch.rand(z.shape, device="cuda") < 0.5] = -math.inf
    s = -rng.uniform(0, float(rng.choice([0.1, 3, 30])), (B, W)).astype(np.float32)
    if rng.random() < 0.2:
        s[:, 1:] = -np.inf
    end = int(rng.integers(-1, V))
    finished = (rng.random((B, W)) < rng.choice([0.2, 0.9])).astype(np.uint8) if end >= 0 and rng.random() < 0.5 else None
    _check(kq, z, s, finished, int(rng.choice([W, rng.integers(1, 33)])), end)


@pytest.mark.parametrize("B", [18, 40, 100, 300])
def test_many_requests(kq, B):
    """Every width of the cluster that the launch picks."""
    for kind, V in ((0, 3001), (2, 1000)):
        _check(kq, _logits(B, B, 8, V, _dtypes()[kind]), _scores(B, B, 8), None, 8, 7)


@pytest.mark.parametrize("kind", [0, 1, 2])
def test_finished_beams_and_the_end_token(kq, kind):
    rng = np.random.default_rng(4)
    logits = _logits(2, 6, 5, 777, _dtypes()[kind])
    logits[:, :, 9] += 9.0                             # the end token is likely
    finished = (rng.random((6, 5)) < 0.5).astype(np.uint8)
    finished[0], finished[1] = 1, 0
    logits[finished == 1] = float("nan")               # not read
    got = _check(kq, logits, _scores(3, 6, 5), finished, 5, 9)
    assert got[3].any() and not got[3].all()
    _check(kq, logits, _scores(3, 6, 5), finished, 11, 9)


def test_masks_dead_beams_and_rows_without_a_distribution(kq):
    import torch
    for dtype in _dtypes():
        lowest = torch.finfo(dtype).min
        z = _logits(5, 9, 4, 600, dtype)
        s = _scores(6, 9, 4)
        z[0, :, 3:] = -math.inf                        # twelve candidates
        z[1] = -math.inf                               # none
        z[2, 1] = lowest                               # a row of the type's lowest value is a flat one
        z[3, :, 5:] = lowest
        z[4, 2, 17] = float("nan")
        z[5, 0, 8] = math.inf
        s[6, 1:] = -math.inf                           # before the first token
        s[7] = [-math.inf, math.nan, math.inf, -2.0]
        s[8] = -math.inf
        for n in (1, 4, 20):
            _check(kq, z, s, None, n, 2)


@pytest.mark.parametrize("B,W,V", [(1, 4, 4099), (70, 5, 700), (400, 16, 90)])
def test_selection_in_place(kq, B, W, V):
    """Scores and ends over those of the step before; another request's inputs may not be read yet."""
    import torch
    z, s = _logits(B, B, W, V, torch.bfloat16), _scores(B, B, W)
    f = (np.random.default_rng(B).random((B, W)) < 0.3).astype(np.uint8)
    want = _check(kq, z, s, f, W, V // 2)
    S, F = torch.from_numpy(s).cuda(), torch.from_numpy(f).cuda()
    p, t = (torch.empty((B, W), dtype=torch.int32, device="cuda") for _ in range(2))
    kq.kvq_beam_select(z, kq.KVQ_BF16, S, F, B, W, V, W, V // 2, p, t, S, F)
    for got, w in zip((p, t, S, F), want):
        assert np.array_equal(got.cpu().numpy(), w)


def test_ties_go_to_the_lowest_beam_and_token(kq):
    import torch
    for dtype in _dtypes():
        for V in (40, 1000, 5001, 20007):
            z = torch.zeros((2, 6, V), dtype=dtype, device="cuda")
            z[1] = (torch.arange(V, device="cuda") % 5).to(dtype)          # many equal maxima
            z[1, :, ::7] = -0.0
            s = np.full((2, 6), -3.0, np.float32)
            parents, tokens, _, _ = _run(kq, z, s, None, 32, -1)
            assert parents[0].tolist() == [0] * 32 and tokens[0].tolist() == list(range(32))
            _check(kq, z, s, None, 32, -1)
    one = _logits(8, 1, 1, 30011, torch.bfloat16, 2.0)
    same = one.repeat(2, 8, 1).contiguous()            # equal rows, of which most are not aligned: exact ties between beams
    parents, tokens, out, _ = _check(kq, same, np.full((2, 8), -1.0, np.float32), None, 32, -1)
    assert parents[0, :8].tolist() == list(range(8)) and len(set(tokens[0, :8].tolist())) == 1 and len(set(out[0, :8].tolist())) == 1


@pytest.mark.parametrize("kind", [0, 2])
def test_sorted_rows(kq, kind):
    """Every chunk holds new best entries, or none."""
    import torch
    up = torch.linspace(-4, 4, 40000, device="cuda")
    z = torch.stack([up, up.flip(0), up.roll(12345)])[None].to(_dtypes()[kind]).contiguous()
    for n in (3, 32):
        _check(kq, z, [[-1.0, -1.5, -2.0]], None, n, -1)


def test_addresses_of_any_alignment(kq):
    import torch
    for dtype in _dtypes():
        flat = _logits(1, 1, 1, 3 * 2 * 4097 + 64, dtype).flatten()
        for shift in range(9):
            _check(kq, flat[shift:shift + 3 * 2 * 4097].reshape(3, 2, 4097), _scores(shift, 3, 2), None, 6, -1)


def test_equal_calls_give_equal_bits_also_in_a_graph(kq):
    import torch
    z, s = _logits(0, 4, 6, 30000, torch.float16), torch.tensor(_scores(0, 4, 6)).cuda()
    outs = [[torch.empty((4, 6), dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32, torch.uint8)] for _ in range(2)]
    call = lambda o: kq.kvq_beam_select(z, kq.KVQ_FP16, s, None, 4, 6, 30000, 6, 2, *o)
    call(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[1])
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*outs))
    z.copy_(_logits(1, 4, 6, 30000, torch.float16))
    graph.replay()
    torch.cuda.synchronize()
    want = _check(kq, z, s.cpu().numpy(), None, 6, 2)
    assert np.array_equal(outs[1][0].cpu().numpy(), want[0]) and np.array_equal(outs[1][1].cpu().numpy(), want[1])


def test_beam_search_over_the_paged_cache(kq):
    """Selection, tables, appended rows and attention as a decoder calls them: a toy model whose logits come from the attention's output, against
    the same search with every beam's rows kept apart in 64 bits."""
    import torch
    rng = np.random.default_rng(3)
    R, W, H, Hq, D, V, page, steps, end = 3, 4, 2, 4, 64, 211, 4, 14, 5
    B, width = R * W, 12
    n_pages = B * width
    emb = [torch.tensor(rng.standard_normal((V, H, D)), dtype=torch.float16).cuda() for _ in range(2)]
    query = torch.tensor(rng.standard_normal((V, Hq, D)), dtype=torch.float16).cuda()
    head = torch.tensor(rng.standard_normal((Hq * D, V)) * 0.5, dtype=torch.float32).cuda()
    K, V_ = [torch.full((n_pages, page, H, D), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2)]
    cache = kq.kvq_page_cache(K, V_)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    tables, lens, cu, copies, status = [i32(B, width), i32(B, width)], i32(B), i32(B + 1), i32(B, 3), i32(1)
    slots, positions = torch.zeros(B, dtype=torch.int64, device="cuda"), i32(B)
    parents, tokens, over = i32(R, W), i32(R, W), torch.zeros((R, W), dtype=torch.uint8, device="cuda")
    scores = torch.full((R, W), -math.inf, device="cuda")
    scores[:, 0] = 0.0
    size = kq.kvq_page_attn_workspace_bytes(B, Hq, H, D)
    work = torch.zeros(size, dtype=torch.uint8, device="cuda")
    O = torch.zeros((B, Hq, D), dtype=torch.float16, device="cuda")
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    tokens.copy_(torch.tensor(rng.integers(0, V, (R, 1))).expand(R, W))
    parents.copy_(torch.arange(B, device="cuda").reshape(R, W))
    hist = [[int(tokens[r, w])] for r in range(R) for w in range(W)]
    for step in range(steps):
        flat = tokens.flatten().long().clamp(min=0)
        kq.kvq_page_step(tables[step % 2], tables[1 - step % 2], width, lens, lens, parents.flatten(), one, B, None, n_pages, page, B, cu, slots,
                         positions, copies, status)
        kq.kvq_page_append(cache, emb[0][flat].contiguous(), emb[1][flat].contiguous(), slots, B, copies, B)
        kq.kvq_page_attn(cache, query[flat].contiguous(), O, None, tables[1 - step % 2], width, lens, B, Hq, D ** -0.5, work, size)
        assert status.item() == 0 and lens.tolist() == [len(h) for h in hist]
        o = O.double().cpu().numpy()
        for b, h in enumerate(hist):                   # the beam's own rows, in 64 bits
            k, v = (e[h].double().cpu().numpy() for e in emb)
            for g in range(H):
                at = slice(g * 2, g * 2 + 2)
                want, _, err, _ = pr.attend(query[h[-1]].double().cpu().numpy()[at], k[:, g], v[:, g], D ** -0.5, 11)
                assert np.all(np.abs(o[b, at] - want) <= err), (step, b, g)
        logits = (O.reshape(B, -1).float() @ head).reshape(R, W, V).contiguous()
        old, ended = scores.cpu().numpy(), over.cpu().numpy()
        new_scores, new_over = torch.empty_like(scores), torch.empty_like(over)
        kq.kvq_beam_select(logits, kq.KVQ_FP32, scores, over, R, W, V, W, end, parents, tokens, new_scores, new_over)
        scores, over = new_scores, new_over
        for r in range(R):
            want = pr.select(logits[r].cpu().numpy(), old[r], ended[r], W, end)
            assert len(want) == W and parents[r].tolist() == [r * W + c[1] for c in want] and tokens[r].tolist() == [c[2] for c in want], (step, r)
        p, t = parents.flatten().tolist(), tokens.flatten().tolist()
        hist = [hist[p[b]] + [t[b]] for b in range(B)]
    distinct = {tuple(h) for h in hist}
    assert len(distinct) == B                          # the beams of a request are different continuations
