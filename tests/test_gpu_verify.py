"""Verification of drafted tokens against the 64-bit reference (GPU): every output is a whole number and has to agree."""
import numpy as np
import pytest

import rows_reference as rr

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_04722_b200 import build
    build.build()
    import gpu_util
    return gpu_util


def _softmax(z):
    e = np.exp(z - z.max(-1, keepdims=True))
    return (e / e.sum(-1, keepdims=True)).astype(np.float32)


def _inputs(seed, B, T, V, chain=False, near=0.7):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((B, T + 1, V)) * 3
    target, draft = _softmax(z), _softmax(z + near * rng.standard_normal(z.shape))
    i = np.arange(T)
    parents = np.tile(i - 1, (B, 1)) if chain else np.maximum(i[None] - rng.integers(1, 4, size=(B, T)), -1)
    tokens = np.empty((B, T), np.int32)
    for b in range(B):
        for k in range(T):
            q = draft[b, parents[b, k] + 1].astype(np.float64)
            tokens[b, k] = rng.choice(V, p=q / q.sum())
    return dict(target=target, draft=draft, tokens=tokens, parents=parents.astype(np.int32),
                u=rng.random((B, T)).astype(np.float32), u_next=rng.random(B).astype(np.float32))


def _run(gu, x, fixed=False):
    import torch
    from paper_2604_04722_b200 import binding as kq
    B, T = x["tokens"].shape
    V = x["target"].shape[2]
    i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, device=gu.DEV)
    acc, path, nxt = i32(B), i32(B, T), i32(B)
    kq.kvq_verify_tree(gu.dev(x["target"]), None if fixed else gu.dev(x["draft"]), gu.dev(x["tokens"]), gu.dev(x["parents"]),
                       B, T, V, gu.dev(x["u"]), gu.dev(x["u_next"]), acc, path, nxt)
    torch.cuda.synchronize()
    return acc.cpu().numpy(), path.cpu().numpy(), nxt.cpu().numpy()


def _check(x, got, fixed=False):
    acc, path, nxt = got
    for b in range(len(acc)):
        want, token = rr.verify(x["target"][b], None if fixed else x["draft"][b], x["tokens"][b], x["parents"][b], x["u"][b],
                                x["u_next"][b])
        assert path[b, :acc[b]].tolist() == want and np.all(path[b, acc[b]:] == -1), (b, path[b], want)
        assert nxt[b] == token, (b, nxt[b], token)


@pytest.mark.parametrize("fixed", [False, True])
@pytest.mark.parametrize("V", [1, 2, 31, 257, 4096, 20011])
@pytest.mark.parametrize("B,T", [(1, 1), (3, 8), (2, 64)])
def test_verification(gu, fixed, V, B, T):
    x = _inputs(V + T, B, T, V)
    _check(x, _run(gu, x, fixed), fixed)


@pytest.mark.parametrize("fixed", [False, True])
@pytest.mark.parametrize("B,V", [(1, 65536), (2, 65537), (1, 150001), (40, 20003)])
def test_vocabularies_that_no_lane_keeps_whole(gu, B, V, fixed):
    """More entries than the registers of the sequence's CTAs hold (65536 at the full width, 8192 at a width of one): the rest of a
    row is read again for every sum."""
    x = _inputs(V, B, 6, V)
    _check(x, _run(gu, x, fixed), fixed)


@pytest.mark.parametrize("B", [40, 80, 200, 700])
def test_many_sequences(gu, B):
    """Every cluster width that the launch picks."""
    for fixed in (False, True):
        x = _inputs(B, B, 5, 300, chain=B % 80 == 0)
        got = _run(gu, x, fixed)
        _check(x, got, fixed)
        assert 0 < got[0].mean() < 5                   # some are accepted, some are turned down


def test_extreme_random_numbers(gu):
    for u, v in ((0.0, 0.0), (1.0 - 2.0 ** -24, 1.0 - 2.0 ** -24), (0.0, 1.0 - 2.0 ** -24), (1.0 - 2.0 ** -24, 0.0)):
        x = _inputs(5, 4, 12, 1000)
        x["u"][:], x["u_next"][:] = np.float32(u), np.float32(v)
        for fixed in (False, True):
            _check(x, _run(gu, x, fixed), fixed)


def test_equal_disjoint_and_one_hot_distributions(gu):
    x = _inputs(6, 3, 10, 500)
    x["draft"] = x["target"].copy()                    # equal: the first child tested is always accepted
    acc, path, nxt = _run(gu, x)
    _check(x, (acc, path, nxt))
    assert np.all(acc >= 1)
    x["target"][:, :, :250], x["draft"][:, :, 250:] = 0, 0     # nothing in common: never accepted
    x["target"] /= x["target"].sum(-1, keepdims=True)
    x["draft"] /= x["draft"].sum(-1, keepdims=True)
    x["tokens"] %= 250
    got = _run(gu, x)
    _check(x, got)
    assert np.all(got[0] == 0) and np.all(got[2] >= 250)
    x["target"][:] = 0                                 # a greedy target: one-hot rows
    x["target"][:, :, 77] = 1
    x["tokens"][:, ::2] = 77
    for fixed in (False, True):
        _check(x, _run(gu, x, fixed), fixed)


def test_rows_without_mass(gu):
    """After a rejection with p <= c q everywhere the next token comes from p; a row of zeros gives -1."""
    x = _inputs(7, 3, 2, 100, chain=True)
    x["draft"][0, 0] = x["target"][0, 0]
    x["u"][0, 0], x["tokens"][0, 0] = np.float32(0.999), 3
    x["target"][0, 0, 3] *= np.float32(0.5)
    x["target"][1] = 0
    _check(x, _run(gu, x))
    _check(x, _run(gu, x, True), True)
    assert _run(gu, x)[2][1] == -1


def test_unused_nodes_duplicates_and_tokens_outside(gu):
    x = _inputs(8, 4, 16, 64)
    x["parents"][:, 5], x["parents"][1, 9], x["parents"][2, 0] = -2, 40, 0
    x["tokens"][:, 1] = x["tokens"][:, 0]              # the same guess twice
    x["tokens"][:, 2], x["tokens"][3, 3] = -1, 64
    x["parents"][:, 1] = x["parents"][:, 2] = -1
    x["u"][0, :2] = np.float32(0.9999)
    for fixed in (False, True):
        _check(x, _run(gu, x, fixed), fixed)


def test_without_nodes_only_the_next_token_is_drawn(gu):
    import torch
    from paper_2604_04722_b200 import binding as kq
    x = _inputs(9, 6, 1, 777)
    target = np.ascontiguousarray(x["target"][:, :1])
    acc = torch.full((6,), 5, dtype=torch.int32, device=gu.DEV)
    nxt = torch.full((6,), -7, dtype=torch.int32, device=gu.DEV)
    kq.kvq_verify_tree(gu.dev(target), None, None, None, 6, 0, 777, None, gu.dev(x["u_next"]), acc, None, nxt)
    assert acc.cpu().tolist() == [0] * 6
    none = np.zeros(0)
    assert nxt.cpu().tolist() == [rr.verify(target[b], None, none, none, none, x["u_next"][b])[1] for b in range(6)]


def test_first_tokens_follow_the_target(gu):
    """20000 sequences with the same distributions: frequencies within five standard deviations."""
    rng = np.random.default_rng(10)
    B, T, V = 20000, 3, 6
    p, q = (rng.dirichlet(np.ones(V)).astype(np.float32) for _ in range(2))
    qn = q.astype(np.float64) / q.sum(dtype=np.float64)
    x = dict(target=np.tile(p, (B, T + 1, 1)), draft=np.tile(q, (B, T + 1, 1)), parents=np.full((B, T), -1, np.int32),
             tokens=rng.choice(V, size=(B, T), p=qn).astype(np.int32), u=rng.random((B, T)).astype(np.float32),
             u_next=rng.random(B).astype(np.float32))
    pn = p.astype(np.float64) / p.sum(dtype=np.float64)
    for fixed in (False, True):
        if fixed:
            x["tokens"][:] = (1, 4, 1)
        acc, path, nxt = _run(gu, x, fixed)
        first = np.where(acc > 0, np.take_along_axis(x["tokens"], np.maximum(path[:, :1], 0), 1)[:, 0], nxt)
        f = np.bincount(first, minlength=V) / B
        assert np.all(np.abs(f - pn) <= 5 * np.sqrt(pn * (1 - pn) / B)), (f, pn)


def test_a_captured_verification(gu):
    import torch
    from paper_2604_04722_b200 import binding as kq
    x, y = _inputs(11, 5, 9, 3000), _inputs(12, 5, 9, 3000)
    want = [_run(gu, v) for v in (x, y)]
    d = {k: gu.dev(v) for k, v in x.items()}
    acc, path, nxt = (torch.zeros(s, dtype=torch.int32, device=gu.DEV) for s in ((5,), (5, 9), (5,)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kq.kvq_verify_tree(d["target"], d["draft"], d["tokens"], d["parents"], 5, 9, 3000, d["u"], d["u_next"], acc, path, nxt)
    for v, w in ((x, want[0]), (y, want[1]), (x, want[0])):
        for k in d:
            d[k].copy_(gu.dev(v[k]))
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip((acc, path, nxt), w))


def test_a_speculative_step_from_draft_to_append(gu, oracle):
    """Tree attention, verification and append as a serving step uses them, twice: the store, the lengths and the
    attention afterwards are those of a cache that only ever saw the accepted rows."""
    import torch
    from paper_2604_04722_b200 import binding as kq
    rng = np.random.default_rng(13)
    B, Hq, H, n, T, V = 3, 6, 2, 90, 10, 400
    widths = np.array([2, 4, 8, 16], np.uint8)
    rows = lambda m: (rng.standard_normal((B, m, H, 64)) * 1.5).astype(np.float16)
    K, Vv, bits = rows(n), rows(n), widths[rng.choice(4, size=(B, n))]
    store = [(K[b], Vv[b], bits[b]) for b in range(B)]
    with gu.GpuCache(1, B, Hq, H, 200) as g:
        g.append(0, K, Vv, bits)
        for step in range(2):
            x = _inputs(20 + step, B, T, V, near=0.3)
            Kd, Vd, bd = rows(T), rows(T), widths[rng.choice(4, size=(B, T))]
            Q = rng.standard_normal((B, T, Hq, 64)).astype(np.float16)
            dK, dV, db, dp = gu.dev(Kd.view(np.uint16)), gu.dev(Vd.view(np.uint16)), gu.dev(bd), gu.dev(x["parents"])
            O = torch.zeros(Q.shape, dtype=torch.float16, device=gu.DEV)
            kq.kvq_attend_tree(g.ctx, 0, gu.dev(Q.view(np.uint16)), dK, dV, db, dp, T, O)
            acc, path, nxt = _run(gu, x)
            _check(x, (acc, path, nxt))
            for b in range(B):                         # what the tree call saw
                oc = oracle.OracleCache(1, Hq, H)
                oc.append(*(a[None] for a in store[b]))
                want, bound = rr.attention(oracle, oc, [len(store[b][0])], Q[b:b + 1], 3,
                                           tree=(Kd[b:b + 1], Vd[b:b + 1], bd[b:b + 1], x["parents"][b:b + 1]))
                assert np.all(np.abs(O[b:b + 1].cpu().numpy().astype(np.float64) - want) <= bound)
            at = torch.from_numpy(np.maximum(path, 0)).long().to(gu.DEV)
            take = lambda t: torch.gather(t, 1, at[:, :, None, None].expand(-1, -1, H, 64)).contiguous()
            kq.kvq_append_ragged(g.ctx, 0, take(dK), take(dV), torch.gather(db, 1, at).contiguous(), None, T, acc)
            for b in range(B):
                p = path[b, :acc[b]]
                store[b] = tuple(np.concatenate([s, d[b][p]]) for s, d in zip(store[b], (Kd, Vd, bd)))
        assert kq.kvq_seq_lens(g.ctx, 0, B).tolist() == [len(s[0]) for s in store]
        m = min(len(s[0]) for s in store)
        got = g.export(0, 0, m)
        for b in range(B):
            oc = oracle.OracleCache(1, Hq, H)
            oc.append(*(a[None] for a in store[b]))
            for k, w in enumerate((oc.bits, oc.pool_slot, oc.kc, oc.vc, oc.km, oc.vm)):
                assert np.array_equal(got[k][b], w[0, :m])
        Q1 = rng.standard_normal((B, 1, Hq, 64)).astype(np.float16)
        O1 = torch.zeros(Q1.shape, dtype=torch.float16, device=gu.DEV)
        kq.kvq_decode_attn_window(g.ctx, 0, gu.dev(Q1.view(np.uint16)), O1, 40, 4)
        for b in range(B):
            oc = oracle.OracleCache(1, Hq, H)
            oc.append(*(a[None] for a in store[b]))
            want, bound = rr.attention(oracle, oc, [len(store[b][0])], Q1[b:b + 1], 3, 40, 4)
            assert np.all(np.abs(O1[b:b + 1].cpu().numpy().astype(np.float64) - want) <= bound)


@pytest.fixture(scope="module")
def drafted():
    return {(V, near): _inputs(V, 6, 9, V, near=near) for V in (50, 5003, 70001) for near in (0.0, 0.7)}


@pytest.mark.parametrize("junk", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("V", [50, 5003, 70001])
def test_draft_rows_that_nothing_was_drawn_from_may_hold_anything(gu, drafted, junk, V):
    """A node without children has no draft distribution, nor has the root of a tree without a node in use.  (The largest
    vocabulary is more than a sequence's registers hold.)"""
    for near in (0.0, 0.7):                            # draft and target equal: leaves are reached
        x = {k: v.copy() for k, v in drafted[V, near].items()}
        x["parents"][0] = -2                           # no node in use: the next token comes from row 0 of the target
        x["parents"][1] = np.arange(9) - 1             # a chain that is accepted as a whole
        x["u"][1] = 0
        for b in range(6):
            drawn = {int(p) + 1 for i, p in enumerate(x["parents"][b]) if -1 <= p < i}
            for row in set(range(10)) - drawn:
                x["draft"][b, row] = junk
        got = _run(gu, x)
        _check(x, got)
        assert got[0][0] == 0 and got[0][1] == 9 and np.all(got[2] >= 0)
