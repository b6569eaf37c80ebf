"""The references of the many-row attention and the draft verification against the oracle and against probability
theory, and the refusals that need no device (CPU)."""
import numpy as np
import pytest

import rows_reference as rr

BITS = np.array([2, 4, 8, 16], np.uint8)


def _cache(oracle, rng, B, n, Hq, H):
    K = (rng.standard_normal((B, n, H, 64)) * 1.5).astype(np.float16)
    V = (rng.standard_normal((B, n, H, 64)) * 1.5).astype(np.float16)
    bits = BITS[rng.choice(4, size=(B, n))]
    oc = oracle.OracleCache(B, Hq, H)
    oc.append(K, V, bits)
    return oc, K, V, bits


def test_window_of_everything_is_the_decode_attention(oracle):
    rng = np.random.default_rng(0)
    oc, _, _, _ = _cache(oracle, rng, 2, 45, 6, 2)
    Q = rng.standard_normal((2, 1, 6, 64)).astype(np.float16)
    want = oc.decode_attn(Q[:, 0]).view(np.float16).astype(np.float64)
    for window, sinks in ((45, 0), (1000, 3), (40, 5)):
        got, bound = rr.attention(oracle, oc, [45, 45], Q, 3, window, sinks)
        assert np.all(np.abs(got[:, 0] - want) <= rr.HALF_STEP * np.abs(want) + 2.0 ** -24)
        assert np.all(bound >= rr.HALF_STEP * np.abs(got))


def test_a_chain_is_the_causal_attention_of_appended_tokens(oracle):
    rng = np.random.default_rng(1)
    n, T = 37, 5
    full, K, V, bits = _cache(oracle, rng, 2, n + T, 4, 2)
    part = oracle.OracleCache(2, 4, 2)
    part.append(K[:, :n], V[:, :n], bits[:, :n])
    Q = rng.standard_normal((2, T, 4, 64)).astype(np.float16)
    parents = np.tile(np.arange(T) - 1, (2, 1)).astype(np.int32)
    want = full.attend_last(Q).view(np.float16).astype(np.float64)
    got, _ = rr.attention(oracle, part, [n, n], Q, 2, tree=(K[:, n:], V[:, n:], bits[:, n:], parents))
    assert np.all(np.abs(got - want) <= rr.HALF_STEP * np.abs(want) + 2.0 ** -24)


def test_siblings_do_not_see_each_other_and_unused_nodes_are_zero(oracle):
    rng = np.random.default_rng(2)
    oc, _, _, _ = _cache(oracle, rng, 1, 9, 2, 2)
    parents = np.array([[-1, -1, 0, -2, 3, 7, 1]], np.int32)
    assert rr.chains(parents[0]) == [[0], [1], [2, 0], None, None, None, [6, 1]]
    K, V = (rng.standard_normal((1, 7, 2, 64)).astype(np.float16) for _ in range(2))
    Q = rng.standard_normal((1, 7, 2, 64)).astype(np.float16)
    base, _ = rr.attention(oracle, oc, [9], Q, 1, tree=(K, V, None, parents))
    K2, V2 = K.copy(), V.copy()
    K2[0, 0] += np.float16(1)
    V2[0, 0] += np.float16(1)
    other, _ = rr.attention(oracle, oc, [9], Q, 1, tree=(K2, V2, None, parents))
    changed = np.any(base != other, axis=(0, 2, 3))
    assert changed.tolist() == [True, False, True, False, False, False, False]
    assert np.all(base[0, 3:6] == 0)


@pytest.mark.parametrize("fixed", [False, True])
def test_verified_tokens_follow_the_target(fixed):
    """The first token that comes out (accepted, or drawn from the residual) has the target's distribution, whatever the
    drafts: 20000 trials, each frequency within five standard deviations."""
    rng = np.random.default_rng(3)
    V, T, n = 6, 3, 20000
    p = rng.dirichlet(np.ones(V)).astype(np.float32)
    q = rng.dirichlet(np.ones(V)).astype(np.float32)
    target = np.tile(p, (T + 1, 1))
    draft = None if fixed else np.tile(q, (T + 1, 1))
    parents = np.full(T, -1)
    hits = np.zeros(V)
    qn = q.astype(np.float64) / q.sum(dtype=np.float64)
    for _ in range(n):
        tokens = np.array([1, 4, 1]) if fixed else rng.choice(V, size=T, p=qn)
        path, nxt = rr.verify(target, draft, tokens, parents, rng.random(T), rng.random())
        hits[tokens[path[0]] if path else nxt] += 1
    pn = p.astype(np.float64) / p.sum(dtype=np.float64)
    assert np.all(np.abs(hits / n - pn) <= 5 * np.sqrt(pn * (1 - pn) / n))


def test_refusals_without_a_device():
    from paper_2604_04722_b200 import build, binding
    build.build()
    L = binding.lib()
    ok = 16
    assert L.kvq_attend_tree(None, 0, ok, ok, ok, None, ok, 1, ok, 0, 0, None) == binding.KVQ_ERR_ARG
    assert L.kvq_decode_attn_window(None, 0, ok, ok, 4, 0, None) == binding.KVQ_ERR_ARG
    verify = lambda **k: L.kvq_verify_tree(*[{**dict(target=ok, draft=None, tokens=ok, parents=ok, batch=1, n=2, vocab=8, u=ok,
                                                     u_next=ok, acc=ok, path=ok, nxt=ok, stream=None), **k}[a]
                                             for a in ("target", "draft", "tokens", "parents", "batch", "n", "vocab", "u", "u_next",
                                                       "acc", "path", "nxt", "stream")])
    for bad in (dict(batch=-1), dict(n=-1), dict(n=binding.KVQ_MAX_TREE_NODES + 1), dict(vocab=0), dict(target=None), dict(tokens=None),
                dict(parents=None), dict(u=None), dict(u_next=None), dict(acc=None), dict(path=None), dict(nxt=None)):
        assert verify(**bad) == binding.KVQ_ERR_ARG, bad
    assert verify(batch=0, target=None) == binding.KVQ_OK


def test_odd_addresses_and_sizes_are_refused_without_a_device():
    from paper_2604_04722_b200 import build, binding
    build.build()
    L = binding.lib()
    names = ("target", "draft", "tokens", "parents", "u", "u_next", "acc", "path", "nxt")

    def verify(vocab=8, **odd):
        p = {**dict.fromkeys(names, 16), **odd}
        return L.kvq_verify_tree(p["target"], p["draft"], p["tokens"], p["parents"], 1, 2, vocab, p["u"], p["u_next"], p["acc"],
                                 p["path"], p["nxt"], None)
    for name in names:
        assert verify(**{name: 18}) == binding.KVQ_ERR_ARG, name
    assert verify(vocab=2 ** 30 + 1) == binding.KVQ_ERR_ARG
