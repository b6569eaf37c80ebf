"""Attention for trees of drafted tokens and windowed decode attention against 64-bit references (GPU)."""
import numpy as np
import pytest

import rows_reference as rr

pytestmark = pytest.mark.gpu

BITS = np.array([2, 4, 8, 16], np.uint8)
MIXED = (.4, .3, .2, .1)


@pytest.fixture(scope="module")
def gu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_04722_b200 import build
    build.build()
    import gpu_util
    return gpu_util


class Case:
    """A cache on both sides: the oracle's rows and a handle with the same tokens (lens per sequence)."""

    def __init__(self, gu, oracle, seed, B, Hq, H, lens, mix=MIXED, bits=None, spread=1.5, value_scale=None):
        rng = np.random.default_rng(seed)
        self.gu, self.oracle, self.rng, self.B, self.Hq, self.H, self.lens = gu, oracle, rng, B, Hq, H, list(lens)
        n = max(max(self.lens), 1)
        K = (rng.standard_normal((B, n, H, 64)) * spread).astype(np.float16)
        V = (rng.standard_normal((B, n, H, 64)) * 1.5).astype(np.float16)
        if value_scale is not None:
            V = (V.astype(np.float64) * value_scale(rng, (B, n, 1, 1))).astype(np.float16)
        bits = BITS[rng.choice(4, size=(B, n), p=mix)] if bits is None else bits(n)[None].repeat(B, 0).astype(np.uint8)
        self.K, self.V, self.bits = K, V, bits
        self.cache = oracle.OracleCache(B, Hq, H)
        self.cache.append(K, V, bits)
        self.g = gu.GpuCache(1, B, Hq, H, n + 80)
        if max(self.lens):
            from paper_2604_04722_b200 import binding as kq
            kq.kvq_append_ragged(self.g.ctx, 0, gu.dev(K.view(np.uint16)), gu.dev(V.view(np.uint16)), gu.dev(bits), None, n,
                                 np.array(self.lens, np.int32))

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.g.close()

    def queries(self, T):
        return self.rng.standard_normal((self.B, T, self.Hq, 64)).astype(np.float16)

    def tree(self, T, kind="tree", with_bits=True):
        rng = self.rng
        K, V = ((rng.standard_normal((self.B, T, self.H, 64)) * 1.5).astype(np.float16) for _ in range(2))
        i = np.arange(T)
        if kind == "chain":
            par = np.tile(i - 1, (self.B, 1))
        elif kind == "star":
            par = np.full((self.B, T), -1)
        else:
            par = np.maximum(i[None] - rng.integers(1, 6, size=(self.B, T)), -1)
        if kind == "ragged":
            for b in range(self.B):
                par[b, max(1, T - 1 - b):] = -2
        bits = BITS[rng.choice(4, size=(self.B, T))] if with_bits else None
        return K, V, bits, par.astype(np.int32)

    def run_tree(self, Q, tree, window=0, sinks=0):
        import torch
        from paper_2604_04722_b200 import binding as kq
        K, V, bits, par = tree
        gu = self.gu
        O = torch.full(Q.shape, 7.0, dtype=torch.float16, device=gu.DEV)
        kq.kvq_attend_tree(self.g.ctx, 0, gu.dev(Q.view(np.uint16)), gu.dev(K.view(np.uint16)), gu.dev(V.view(np.uint16)),
                           None if bits is None else gu.dev(bits), gu.dev(par), Q.shape[1], O, window, sinks)
        torch.cuda.synchronize()
        assert kq.kvq_device_status(self.g.ctx) == 0
        return O.cpu().numpy()

    def run_window(self, Q, window, sinks):
        import torch
        from paper_2604_04722_b200 import binding as kq
        O = torch.full(Q.shape, 7.0, dtype=torch.float16, device=self.gu.DEV)
        kq.kvq_decode_attn_window(self.g.ctx, 0, self.gu.dev(Q.view(np.uint16)), O, window, sinks)
        torch.cuda.synchronize()
        assert kq.kvq_device_status(self.g.ctx) == 0
        return O.cpu().numpy()

    def check(self, got, Q, window=0, sinks=0, tree=None):
        want, bound = rr.attention(self.oracle, self.cache, self.lens, Q, self.Hq // self.H, window, sinks, tree)
        err = np.abs(got.astype(np.float64).reshape(want.shape) - want)
        worst = np.unravel_index(np.argmax(err - bound), err.shape)
        assert np.all(err <= bound), "at %s: got %g want %g, off by %.3e, bound %.3e" % (
            worst, got.reshape(want.shape)[worst], want[worst], err[worst], bound[worst])


@pytest.mark.parametrize("n", [1, 15, 16, 17, 33, 257, 700])
@pytest.mark.parametrize("Hq,H", [(1, 1), (6, 2), (8, 1)])
def test_tree_over_a_cache(gu, oracle, n, Hq, H):
    with Case(gu, oracle, n + Hq, 2, Hq, H, [n, n]) as c:
        for T, kind in ((1, "tree"), (7, "tree"), (16, "chain"), (17, "ragged")):
            Q, t = c.queries(T), c.tree(T, kind)
            c.check(c.run_tree(Q, t), Q, tree=t)


@pytest.mark.parametrize("T", [2, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("group", [1, 3])
def test_tree_sizes(gu, oracle, T, group):
    with Case(gu, oracle, T, 1, 2 * group, 2, [130]) as c:
        for kind, with_bits in (("tree", True), ("chain", False), ("star", True)):
            Q, t = c.queries(T), c.tree(T, kind, with_bits)
            c.check(c.run_tree(Q, t), Q, tree=t)


@pytest.mark.parametrize("Hq,H", [(15, 1), (16, 1), (17, 1), (40, 2)])
def test_tree_group_sizes(gu, oracle, Hq, H):
    with Case(gu, oracle, Hq, 1, Hq, H, [90]) as c:
        for T in (1, 3):
            Q, t = c.queries(T), c.tree(T)
            c.check(c.run_tree(Q, t), Q, tree=t)


@pytest.mark.parametrize("b", [2, 4, 8, 16])
@pytest.mark.parametrize("n", [1, 16, 2000])
def test_tree_over_one_precision(gu, oracle, b, n):
    """2000 tokens of one class pass the border of a 64 KB block (1600 / 880 / 480 / 256 tokens)."""
    with Case(gu, oracle, b + n, 1, 3, 1, [n], bits=lambda m: np.full(m, b)) as c:
        Q, t = c.queries(5), c.tree(5)
        c.check(c.run_tree(Q, t), Q, tree=t)
        c.check(c.run_tree(Q, t, 1700, 3), Q, 1700, 3, t)
        Q1 = c.queries(1)
        c.check(c.run_window(Q1, 1111, 2), Q1, 1111, 2)


def test_tree_over_an_empty_cache(gu, oracle):
    with Case(gu, oracle, 5, 2, 4, 2, [0, 0]) as c:
        for kind in ("tree", "ragged", "chain"):
            Q, t = c.queries(9), c.tree(9, kind)
            c.check(c.run_tree(Q, t), Q, tree=t)
            c.check(c.run_tree(Q, t, 2, 1), Q, 2, 1, t)


def test_tree_and_window_on_ragged_lengths(gu, oracle):
    with Case(gu, oracle, 6, 5, 6, 2, [0, 1, 300, 17, 299]) as c:
        for window, sinks in ((0, 0), (1, 0), (16, 3), (250, 20)):
            Q, t = c.queries(21), c.tree(21, "ragged")
            c.check(c.run_tree(Q, t, window, sinks), Q, window, sinks, t)
            if window:
                Q1 = c.queries(1)
                got = c.run_window(Q1, window, sinks)
                c.check(got, Q1, window, sinks)
                assert np.all(got[0] == 0)


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 64, 100, 499, 500, 501, 2 ** 31 - 1])
@pytest.mark.parametrize("sinks", [0, 1, 4, 33, 600])
def test_windows_and_sinks(gu, oracle, window, sinks):
    with Case(gu, oracle, 7, 2, 6, 2, [500, 500]) as c:
        Q = c.queries(1)
        c.check(c.run_window(Q, window, sinks), Q, window, sinks)
        if sinks in (0, 4) or window < 20:
            Q, t = c.queries(12), c.tree(12, "chain")
            c.check(c.run_tree(Q, t, window, sinks), Q, window, sinks, t)


@pytest.mark.parametrize("window", [3, 40, 700])
def test_deep_chain_with_its_own_tokens_leaving_the_window(gu, oracle, window):
    with Case(gu, oracle, 8, 1, 2, 1, [100]) as c:
        Q, t = c.queries(64), c.tree(64, "chain")
        for sinks in (0, 2, 100, 130):                 # the sinks may reach into the drafted positions
            c.check(c.run_tree(Q, t, window, sinks), Q, window, sinks, t)


@pytest.mark.parametrize("where", ["first", "last", "none"])
def test_window_when_a_class_is_rare(gu, oracle, where):
    """A class with one token at the start or the end of a long sequence, far from where the window starts."""
    def bits(m):
        x = np.full(m, 4)
        if where == "first":
            x[0], x[1] = 2, 16
        elif where == "last":
            x[-1], x[-2] = 8, 16
        return x
    with Case(gu, oracle, 9, 1, 3, 1, [1500], bits=bits) as c:
        Q, t = c.queries(6), c.tree(6)
        for window, sinks in ((900, 0), (1300, 1), (7, 2), (2, 1)):
            Q1 = c.queries(1)
            c.check(c.run_window(Q1, window, sinks), Q1, window, sinks)
            c.check(c.run_tree(Q, t, window, sinks), Q, window, sinks, t)


@pytest.mark.parametrize("B,Hq,H,n,T", [(1, 3, 1, 9000, 20), (3, 6, 2, 5000, 4), (1, 1, 1, 20000, 64)])
def test_parts_of_a_unit_are_merged(gu, oracle, B, Hq, H, n, T):
    """Few units and long caches: a unit is cut into several CTAs."""
    with Case(gu, oracle, n, B, Hq, H, [n] * B) as c:
        Q, t = c.queries(T), c.tree(T)
        got = c.run_tree(Q, t)
        c.check(got, Q, tree=t)
        assert np.array_equal(got, c.run_tree(Q, t))   # the parts are merged in order: the same bits again
        Q1 = c.queries(1)
        c.check(c.run_window(Q1, n - 100, 4), Q1, n - 100, 4)


def test_peaked_and_wide_ranged_inputs(gu, oracle):
    """Logits far apart, and value scales from 2^-12 to 2^10 per token."""
    scale = lambda rng, shape: 2.0 ** rng.integers(-12, 11, size=shape)
    with Case(gu, oracle, 11, 1, 4, 2, [400], spread=12.0, value_scale=scale) as c:
        for f in (0.01, 1.0, 20.0):
            Q = (c.queries(9).astype(np.float32) * f).astype(np.float16)
            t = c.tree(9)
            c.check(c.run_tree(Q, t), Q, tree=t)
            Q1 = (c.queries(1).astype(np.float32) * f).astype(np.float16)
            c.check(c.run_window(Q1, 200, 4), Q1, 200, 4)


def test_rows_of_very_different_queries(gu, oracle):
    """Rows of one block whose queries differ by 2^20, and a row of zeros."""
    with Case(gu, oracle, 12, 1, 4, 1, [333]) as c:
        Q, t = c.queries(4).astype(np.float32), c.tree(4)
        Q *= (2.0 ** np.array([-12, 0, 5, 8]))[None, :, None, None]
        Q[0, 2, 1] = 0
        Q = Q.astype(np.float16)
        c.check(c.run_tree(Q, t), Q, tree=t)


def test_degenerate_drafted_rows(gu, oracle):
    """Constant rows, zeros, signed zeros, subnormal scales, the largest fp16 values."""
    with Case(gu, oracle, 13, 1, 2, 1, [20]) as c:
        T = 12
        Q = c.queries(T)
        K, V, _, par = c.tree(T, "star")
        K[0, 0], V[0, 0] = 0, 0
        V[0, 1] = np.float16(3.25)
        V[0, 2, :, ::2] = np.float16(-0.0)
        V[0, 3] = (V[0, 3].astype(np.float64) * 2.0 ** -22).astype(np.float16)
        V[0, 4], V[0, 4, :, 3] = np.float16(-65504), np.float16(65504)
        Q[0, 4] = 0
        for b in (2, 4, 8, 16):
            t = (K, V, np.full((1, T), b, np.uint8), par)
            c.check(c.run_tree(Q, t), Q, tree=t)


def test_garbage_in_unused_nodes_stays_out(gu, oracle):
    with Case(gu, oracle, 14, 2, 6, 2, [50, 50]) as c:
        Q, (K, V, bits, par) = c.queries(20), c.tree(20, "ragged")
        par[0, 3], par[1, 5] = 3, 100                  # not an earlier node
        want = c.run_tree(Q, (K, V, bits, par))
        for b in range(2):
            for i, ch in enumerate(rr.chains(par[b])):
                if ch is None:
                    K[b, i], V[b, i], Q[b, i] = np.nan, np.inf, np.nan
                    assert np.all(want[b, i] == 0)
        clean = Q.copy()
        clean[np.isnan(clean)] = 0
        got = c.run_tree(clean, (K, V, bits, par))
        assert np.array_equal(got, want)


@pytest.mark.parametrize("junk", [np.nan, np.inf, -65504.0])
def test_queries_of_unused_nodes_stay_out(gu, oracle, junk):
    """Their rows share blocks with rows in use."""
    with Case(gu, oracle, 24, 2, 6, 2, [60, 60]) as c:
        Q, t = c.queries(13), c.tree(13, "ragged")
        for b in range(2):
            for i, ch in enumerate(rr.chains(t[3][b])):
                if ch is None:
                    Q[b, i] = np.float16(junk)
        clean = Q.copy()
        for b in range(2):
            for i, ch in enumerate(rr.chains(t[3][b])):
                if ch is None:
                    clean[b, i] = 0
        c.check(c.run_tree(Q, t), clean, tree=t)


@pytest.mark.parametrize("splits", [1, 5, 16, 64])
def test_explicit_splits(gu, oracle, splits):
    from paper_2604_04722_b200 import binding as kq
    with Case(gu, oracle, 25, 2, 6, 2, [700, 650]) as c:
        kq.kvq_set_splits(c.g.ctx, splits)
        for T in (1, 6, 30):
            Q, t = c.queries(T), c.tree(T)
            c.check(c.run_tree(Q, t), Q, tree=t)
        Q1 = c.queries(1)
        c.check(c.run_window(Q1, 400, 4), Q1, 400, 4)


@pytest.mark.parametrize("B,Hq,H,n,T", [(40, 32, 32, 300, 1), (13, 30, 10, 900, 9), (3, 32, 32, 2300, 12), (20, 32, 32, 60, 3)])
def test_many_units(gu, oracle, B, Hq, H, n, T):
    """More units than CTAs fit the device: whole units, and stretches of the axis that cross unit borders.  Three sequences
    of the batch are compared."""
    rng = np.random.default_rng(n)
    import torch
    from paper_2604_04722_b200 import binding as kq
    with Case(gu, oracle, n, B, Hq, H, [n] * B) as c:
        Q, t = c.queries(T), c.tree(T)
        got, Q1 = c.run_tree(Q, t, n - 30, 2), c.queries(1)
        got1 = c.run_window(Q1, n - 7, 3)
        for b in (0, B // 2, B - 1):
            part = oracle.OracleCache(1, Hq, H)
            part.append(c.K[b:b + 1], c.V[b:b + 1], c.bits[b:b + 1])
            sub = tuple(x[b:b + 1] for x in t)
            for out, q, kw in ((got, Q, dict(window=n - 30, sinks=2, tree=sub)), (got1, Q1, dict(window=n - 7, sinks=3))):
                want, bound = rr.attention(oracle, part, [n], q[b:b + 1], Hq // H, **kw)
                assert np.all(np.abs(out[b:b + 1].astype(np.float64).reshape(want.shape) - want) <= bound)


def test_long_ragged_batch_over_the_whole_axis(gu, oracle):
    """Lengths from nothing to long, so that some stretches of the axis are empty."""
    with Case(gu, oracle, 26, 6, 6, 2, [2500, 0, 1, 2100, 16, 900]) as c:
        for T in (2, 8, 40):
            Q, t = c.queries(T), c.tree(T, "ragged")
            c.check(c.run_tree(Q, t), Q, tree=t)
        Q1 = c.queries(1)
        c.check(c.run_window(Q1, 2000, 4), Q1, 2000, 4)


def test_long_caches_keep_the_precision_of_short_ones(gu, oracle):
    """60000 tokens in one CTA.  The roundings of the weights to fp16 are independent and each is uniform within 2^-11 of its
    value at most, so next to the outputs, which are the same sums of values of random sign, they are off by 2^-11 / sqrt(3) in
    the mean square; the rounding of the output is as much again at most: together 4.0e-4, whatever the length."""
    from paper_2604_04722_b200 import binding as kq
    with Case(gu, oracle, 28, 1, 3, 1, [60000]) as c:
        kq.kvq_set_splits(c.g.ctx, 4)
        Q, t = c.queries(4), c.tree(4)
        got = c.run_tree(Q, t).astype(np.float64)
        want, _ = rr.attention(oracle, c.cache, c.lens, Q, 3, tree=t)
        assert np.linalg.norm(got - want) <= 2.0 ** -11 * (2 / 3) ** .5 * np.linalg.norm(want)


def test_stale_blocks_of_an_earlier_cache_stay_out(gu, oracle):
    """Blocks that held huge fp16 rows are handed out again after a reset."""
    import torch
    from paper_2604_04722_b200 import binding as kq
    rng = np.random.default_rng(15)
    with Case(gu, oracle, 15, 1, 2, 1, [21], mix=(.1, .1, .1, .7)) as c:
        kq.kvq_reset(c.g.ctx)
        junk = np.full((1, 90, 1, 64), np.inf, np.float16)
        full = np.full((1, 90), 16, np.uint8)
        c.g.append(0, junk, junk, full)
        kq.kvq_reset(c.g.ctx)
        c.g.append(0, c.K, c.V, c.bits)
        Q, t = c.queries(3), c.tree(3)
        c.check(c.run_tree(Q, t), Q, tree=t)
        Q1 = c.queries(1)
        c.check(c.run_window(Q1, 9, 1), Q1, 9, 1)


@pytest.mark.parametrize("b", [2, 4, 8, 16])
@pytest.mark.parametrize("pattern", [0x7c00, 0xffff])
def test_slots_without_a_token_may_hold_any_bytes(gu, oracle, b, pattern):
    """Blocks that held rows of Inf or NaN patterns, whatever the pool that gets them next."""
    from paper_2604_04722_b200 import binding as kq
    with Case(gu, oracle, b, 1, 2, 1, [21], bits=lambda m: np.full(m, b)) as c:
        kq.kvq_reset(c.g.ctx)
        junk = np.full((1, 100, 1, 64), pattern, np.uint16).view(np.float16)
        c.g.append(0, junk, junk, np.full((1, 100), 16, np.uint8))
        kq.kvq_reset(c.g.ctx)
        c.g.append(0, c.K, c.V, c.bits)
        Q, t = c.queries(3), c.tree(3)
        c.check(c.run_tree(Q, t), Q, tree=t)
        Q1 = c.queries(1)
        c.check(c.run_window(Q1, 9, 1), Q1, 9, 1)


@pytest.mark.parametrize("b", [2, 4, 8, 16])
@pytest.mark.parametrize("bad", [np.inf, np.nan])
def test_cached_tokens_that_nobody_sees_may_hold_anything(gu, oracle, b, bad):
    with Case(gu, oracle, b, 1, 4, 2, [150], bits=lambda m: np.full(m, b)) as c:
        Q1, Q, t = c.queries(1), c.queries(7), c.tree(7, "star")
        at = slice(5, 150 - 41)                        # neither among 5 sinks nor in a window of 40
        dirty = Case(gu, oracle, b, 1, 4, 2, [0], bits=lambda m: np.full(m, b))
        dirty.g.close()
        dirty.g = gu.GpuCache(1, 1, 4, 2, 300)
        K, V = c.K.copy(), c.V.copy()
        K[:, at], V[:, at] = bad, bad
        dirty.g.append(0, K, V, c.bits)
        # The append lets a quantized row that is not finite reach the codes of a neighbour; the attention is held to what
        # is stored.
        _, _, kc, vc, km, vm = dirty.g.export(0, 0, 150)
        seen = np.r_[0:5, 109:150]
        for mine, stored in ((c.cache.kc, kc), (c.cache.vc, vc), (c.cache.km, km), (c.cache.vm, vm)):
            mine[:, seen] = stored[:, seen].reshape(mine[:, seen].shape)
        c.check(dirty.run_window(Q1, 40, 5), Q1, 40, 5)
        c.check(dirty.run_tree(Q, t, 41, 5), Q, 41, 5, t)
        dirty.g.close()


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_a_drafted_row_that_is_not_finite_concerns_its_descendants_only(gu, oracle, bad):
    with Case(gu, oracle, 27, 1, 6, 2, [70]) as c:
        T, hit = 22, (3, 17)
        Q, (K, V, bits, par) = c.queries(T), c.tree(T)
        bits[0, list(hit)] = 16
        want, bound = rr.attention(oracle, c.cache, c.lens, Q, 3, tree=(K.copy(), V.copy(), bits, par))
        V[0, list(hit), :, 5] = bad
        K[0, 17] = bad
        got = c.run_tree(Q, (K, V, bits, par))
        for i, ch in enumerate(rr.chains(par[0])):
            if set(ch) & set(hit):
                assert not np.any(np.isfinite(got[0, i]))
            else:
                assert np.all(np.abs(got[0, i].astype(np.float64) - want[0, i]) <= bound[0, i])


def test_bad_bits_are_flagged_and_kept_as_fp16(gu, oracle):
    import torch
    from paper_2604_04722_b200 import binding as kq
    with Case(gu, oracle, 16, 1, 2, 1, [30]) as c:
        Q, (K, V, bits, par) = c.queries(4), c.tree(4)
        bits[0, 1] = 16
        want = c.run_tree(Q, (K, V, bits, par))
        bits[0, 1] = 5
        O = torch.zeros(Q.shape, dtype=torch.float16, device=gu.DEV)
        kq.kvq_attend_tree(c.g.ctx, 0, gu.dev(Q.view(np.uint16)), gu.dev(K.view(np.uint16)), gu.dev(V.view(np.uint16)),
                           gu.dev(bits), gu.dev(par), 4, O)
        assert kq.kvq_device_status(c.g.ctx) == 1      # KVQ_FLAG_BAD_BITS
        assert np.array_equal(O.cpu().numpy(), want)


def test_a_chain_equals_appending_it(gu, oracle):
    """The same rows drafted as a chain, and appended and asked through kvq_attend_last; the drafted call leaves the
    cache alone."""
    with Case(gu, oracle, 17, 2, 6, 2, [333, 333]) as c:
        T = 11
        Q, t = c.queries(T), c.tree(T, "chain")
        got = c.run_tree(Q, t)
        gu.assert_store_equals_oracle(c.g, 0, c.cache)
        c.g.append(0, t[0], t[1], t[2])
        import torch
        from paper_2604_04722_b200 import binding as kq
        O = torch.zeros(Q.shape, dtype=torch.float16, device=gu.DEV)
        kq.kvq_attend_last(c.g.ctx, 0, gu.dev(Q.view(np.uint16)), O, T)
        want, bound = rr.attention(oracle, c.cache, c.lens, Q, 3, tree=t)
        err = np.abs(got.astype(np.float64) - O.cpu().numpy().astype(np.float64))
        assert np.all(err <= bound + rr.HALF_STEP * np.abs(want) * 2 + 1e-5)   # both sides' output roundings


def test_a_window_of_everything_equals_the_decode_attention(gu, oracle):
    with Case(gu, oracle, 18, 3, 6, 2, [700] * 3) as c:
        Q = c.queries(1)
        got = c.run_window(Q, 5000, 0)
        ref = c.g.decode(0, Q[:, 0]).view(np.float16).astype(np.float64)
        _, bound = rr.attention(oracle, c.cache, c.lens, Q, 3)
        assert np.all(np.abs(got[:, 0].astype(np.float64) - ref) <= bound[:, 0] + 2 * rr.HALF_STEP * np.abs(ref) + 1e-5)


def test_another_stream_and_a_captured_graph(gu, oracle):
    import torch
    from paper_2604_04722_b200 import binding as kq
    with Case(gu, oracle, 19, 1, 3, 1, [6000]) as c:    # cut into several CTAs: the arrival counters have to come back
        Q, t = c.queries(8), c.tree(8)
        want_t, Q1 = c.run_tree(Q, t, 900, 2), c.queries(1)
        want_w = c.run_window(Q1, 3000, 4)
        dq, dk, dv = (gu.dev(a.view(np.uint16)) for a in (Q, t[0], t[1]))
        db, dp, dq1 = gu.dev(t[2]), gu.dev(t[3]), gu.dev(Q1.view(np.uint16))
        O = torch.zeros(Q.shape, dtype=torch.float16, device=gu.DEV)
        O1 = torch.zeros(Q1.shape, dtype=torch.float16, device=gu.DEV)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            kq.kvq_attend_tree(c.g.ctx, 0, dq, dk, dv, db, dp, 8, O, 900, 2)
            kq.kvq_decode_attn_window(c.g.ctx, 0, dq1, O1, 3000, 4)
        side.synchronize()
        assert np.array_equal(O.cpu().numpy(), want_t) and np.array_equal(O1.cpu().numpy(), want_w)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kq.kvq_attend_tree(c.g.ctx, 0, dq, dk, dv, db, dp, 8, O, 900, 2)
            kq.kvq_decode_attn_window(c.g.ctx, 0, dq1, O1, 3000, 4)
        for _ in range(3):
            O.zero_()
            O1.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert np.array_equal(O.cpu().numpy(), want_t) and np.array_equal(O1.cpu().numpy(), want_w)


def test_refusals(gu, oracle):
    import torch
    from paper_2604_04722_b200 import binding as kq
    with Case(gu, oracle, 20, 1, 2, 1, [10]) as c:
        h = lambda *s: torch.zeros(s, dtype=torch.float16, device=gu.DEV)
        Q, K, V, O = h(1, 4, 2, 64), h(1, 4, 1, 64), h(1, 4, 1, 64), h(1, 4, 2, 64)
        odd = torch.zeros(4 * 2 * 64 + 8, dtype=torch.float16, device=gu.DEV)[1:1 + 4 * 2 * 64]
        par = torch.full((1, 4), -1, dtype=torch.int32, device=gu.DEV)

        def tree(**k):
            a = {**dict(layer=0, Q=Q, K=K, V=V, bits=None, par=par, n=4, O=O, window=0, sinks=0), **k}
            kq.kvq_attend_tree(c.g.ctx, a["layer"], a["Q"], a["K"], a["V"], a["bits"], a["par"], a["n"], a["O"], a["window"], a["sinks"])

        def window(**k):
            a = {**dict(layer=0, Q=Q, O=O, window=4, sinks=0), **k}
            kq.kvq_decode_attn_window(c.g.ctx, a["layer"], a["Q"], a["O"], a["window"], a["sinks"])

        for bad in (dict(layer=1), dict(layer=-1), dict(n=65), dict(n=-1), dict(window=-1), dict(sinks=-1), dict(Q=None), dict(K=None),
                    dict(V=None), dict(par=None), dict(O=None), dict(Q=odd), dict(O=odd), dict(K=odd), dict(V=odd)):
            with pytest.raises(kq.KvqError) as e:
                tree(**bad)
            assert e.value.code == kq.KVQ_ERR_ARG, bad
        with pytest.raises(kq.KvqError) as e:          # int32 at an odd address
            tree(par=torch.zeros(20, dtype=torch.int8, device=gu.DEV)[1:17])
        assert e.value.code == kq.KVQ_ERR_ARG
        O.fill_(3.0)
        tree(n=0, Q=None)                              # nothing to do
        assert torch.all(O == 3.0)
        for bad in (dict(layer=1), dict(window=0), dict(window=-3), dict(sinks=-1), dict(Q=None), dict(O=None), dict(Q=odd), dict(O=odd)):
            with pytest.raises(kq.KvqError) as e:
                window(**bad)
            assert e.value.code == kq.KVQ_ERR_ARG, bad
        kq.kvq_reset(c.g.ctx)
        with pytest.raises(kq.KvqError) as e:
            window()
        assert e.value.code == kq.KVQ_ERR_EMPTY
    for other in (dict(scale_groups=2), dict(k_per_channel=True)):
        with gu.GpuCache(1, 1, 2, 1, 64, **other) as g:
            for call in (lambda: kq.kvq_attend_tree(g.ctx, 0, Q, K, V, None, par, 4, O),
                         lambda: kq.kvq_decode_attn_window(g.ctx, 0, Q, O, 4)):
                with pytest.raises(kq.KvqError) as e:
                    call()
                assert e.value.code == kq.KVQ_ERR_ARG


@pytest.mark.parametrize("b", [2, 4, 8])
@pytest.mark.parametrize("where", ["K", "V"])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_one_bad_channel_of_a_drafted_row_that_is_stored_quantized(gu, oracle, b, where, bad):
    """Such a row has no finite values (its scale or its zero-point is not finite): those who see it become NaN, whatever the
    width, and nobody else does."""
    with Case(gu, oracle, 30 + b, 2, 6, 2, [70, 33]) as c:
        T, hit = 22, (3, 17)
        Q, (K, V, bits, par) = c.queries(T), c.tree(T)
        bits[:, list(hit)] = b
        want, bound = rr.attention(oracle, c.cache, c.lens, Q, 3, tree=(K.copy(), V.copy(), bits, par))
        (K if where == "K" else V)[:, list(hit), :, 5] = bad
        got = c.run_tree(Q, (K, V, bits, par))
        for s in range(2):
            for i, ch in enumerate(rr.chains(par[s])):
                if set(ch) & set(hit):
                    assert np.all(np.isnan(got[s, i])), (s, i)
                else:
                    assert np.all(np.abs(got[s, i].astype(np.float64) - want[s, i]) <= bound[s, i]), (s, i)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("with_bits", [False, True])
def test_one_bad_channel_of_a_drafted_key_that_stays_fp16(gu, oracle, bad, with_bits):
    """The softmax as it stands: a logit of minus infinity has the weight zero, any other that is not finite makes NaN."""
    with Case(gu, oracle, 36, 1, 6, 2, [70]) as c:
        T, hit = 22, 3
        Q, (K, V, bits, par) = c.queries(T), c.tree(T, with_bits=with_bits)
        if with_bits:
            bits[0, hit] = 16
        want, bound = rr.attention(oracle, c.cache, c.lens, Q, 3, tree=(K.copy(), V.copy(), bits, par))
        past = par.copy()                              # the same tree with that node out of everybody's chain
        past[0, par[0] == hit] = par[0, hit]
        without, bound_without = rr.attention(oracle, c.cache, c.lens, Q, 3, tree=(K.copy(), V.copy(), bits, past))
        K[0, hit, :, 5] = bad
        got = c.run_tree(Q, (K, V, bits, par))
        zero = Q[0, :, :, 5].astype(np.float64) * bad == -np.inf
        assert np.isnan(bad) or (np.any(zero) and not np.all(zero))
        for i, ch in enumerate(rr.chains(par[0])):
            for h in range(6):
                if hit not in ch:
                    assert np.all(np.abs(got[0, i, h].astype(np.float64) - want[0, i, h]) <= bound[0, i, h])
                elif not zero[i, h]:
                    assert np.all(np.isnan(got[0, i, h])), (i, h)
                elif i != hit:
                    assert np.all(np.abs(got[0, i, h].astype(np.float64) - without[0, i, h]) <= bound_without[0, i, h]), (i, h)


@pytest.mark.parametrize("junk", [0, 3, 255])
def test_bit_widths_of_unused_nodes_may_be_anything(gu, oracle, junk):
    """A padded tree is no error: no flag (run_tree asserts that), no change.  A node in use with the same width is one."""
    import torch
    from paper_2604_04722_b200 import binding as kq
    with Case(gu, oracle, 31, 2, 6, 2, [50, 0]) as c:
        Q, (K, V, bits, par) = c.queries(40), c.tree(40, "ragged")
        par[0, 4], par[1, 7] = 4, 100                  # not an earlier node, and their descendants with them
        want = c.run_tree(Q, (K, V, bits, par))
        unused = np.array([[ch is None for ch in rr.chains(par[b])] for b in range(2)])
        assert np.any(unused[:, :32]) and np.any(unused[:, 32:])
        padded = np.where(unused, np.uint8(junk), bits)
        assert np.array_equal(c.run_tree(Q, (K, V, padded, par)), want)
        for i in (0, 33):                              # one in use in each half of the nodes
            spoiled = padded.copy()
            par[1, i] = -1
            spoiled[1, i] = junk
            O = torch.zeros(Q.shape, dtype=torch.float16, device=gu.DEV)
            kq.kvq_attend_tree(c.g.ctx, 0, gu.dev(Q.view(np.uint16)), gu.dev(K.view(np.uint16)), gu.dev(V.view(np.uint16)),
                               gu.dev(spoiled), gu.dev(par), 40, O)
            assert kq.kvq_device_status(c.g.ctx) == 1  # KVQ_FLAG_BAD_BITS


@pytest.mark.parametrize("junk", [65504.0, np.inf, np.nan])
@pytest.mark.parametrize("window", [0, 50])
def test_large_queries_of_unused_nodes_cost_the_others_no_bits(gu, oracle, junk, window):
    """Small queries over large keys, next to unused rows of the largest values: the same bits as with zeros there."""
    with Case(gu, oracle, 32, 2, 6, 2, [90, 75], spread=2.0 ** 10) as c:
        Q, (K, V, bits, par) = c.queries(13), c.tree(13, "ragged")
        par[0, 2] = 2                                  # and its descendants
        Q = (Q.astype(np.float32) * 2.0 ** -10).astype(np.float16)
        unused = np.array([[ch is None for ch in rr.chains(par[b])] for b in range(2)])
        Q[unused] = 0
        want = c.run_tree(Q, (K, V, bits, par), window)
        c.check(want, Q, window, tree=(K, V, bits, par))
        Q[unused] = np.float16(junk)
        got = c.run_tree(Q, (K, V, bits, par), window)
        assert np.array_equal(got, want)
        assert np.all(got[unused] == 0)


def test_layouts_that_refuse_these_calls_hold_no_memory_for_them(gu):
    """The partial records (256 bytes for each of 128 rows per SM, and their counters) are part of handles with one scale group."""
    import torch
    from paper_2604_04722_b200 import binding as kq
    records = torch.cuda.get_device_properties(0).multi_processor_count * 128 * 256
    arena = 40 * 65536
    need = [kq.kvq_workspace_bytes(1, 2, 1, 64, 64, 1, arena, groups) for groups in (1, 2)]
    assert need[0] - need[1] >= records
    handles = [kq.kvq_create_arena(1, 2, 1, 64, 64, 1, arena), kq.kvq_create_grouped(1, 2, 1, 64, 64, 1, arena, 2),
               kq.kvq_create_perchannel(1, 2, 1, 64, 64, 1, arena)]
    held = [kq.kvq_device_bytes(h) for h in handles]
    assert held[0] - held[1] >= records and held[0] - held[2] >= records - 2 ** 16   # (waiting rows of per-channel keys)
    for h in handles:
        kq.kvq_recover(h)
        kq.kvq_destroy(h)
