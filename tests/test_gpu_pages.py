"""The paged 16-bit cache against plain definitions in 64 bits (GPU)."""
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


# ---------------------------------------------------------------- tables and slots

class Step:
    """Buffers of a step; run() returns what the kernel wrote as numpy arrays."""

    def __init__(self, kq, tables, lens, parents, new, held, n_pages, page, max_new, in_place=False):
        import torch
        t = lambda a, dt=torch.int32: None if a is None else torch.as_tensor(np.ascontiguousarray(a), dtype=dt).cuda()
        self.kq, self.B, self.args = kq, len(lens), (n_pages, page, max_new)
        self.tables, self.lens, self.parents, self.new, self.held = t(tables), t(lens), t(parents), t(new), t(held, torch.uint8)
        i32 = lambda *s: torch.full(s, -77, dtype=torch.int32, device="cuda")
        self.out = dict(tables=self.tables if in_place else i32(*self.tables.shape), lens=self.lens if in_place else i32(self.B), cu=i32(self.B + 1),
                        slots=torch.full((max_new,), -77, dtype=torch.int64, device="cuda"), positions=i32(max_new), copies=i32(self.B, 3), status=i32(1))

    def call(self):
        n_pages, page, max_new = self.args
        o = self.out
        self.kq.kvq_page_step(self.tables, o["tables"], self.tables.shape[1], self.lens, o["lens"], self.parents, self.new, self.B, self.held,
                              n_pages, page, max_new, o["cu"], o["slots"], o["positions"], o["copies"], o["status"])

    def run(self):
        import torch
        self.call()
        torch.cuda.synchronize()
        return {k: v.cpu().numpy() for k, v in self.out.items()}


def _state(seed, B, page, longest, n_pages, width, groups=1):
    """Tables of rows of random lengths; rows of a group share their first full pages."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, longest + 1, B)
    order, at = rng.permutation(n_pages), 0
    tables = rng.integers(-5, 10 ** 9, (B, width)).astype(np.int64)        # behind a row's pages anything may stand
    for b in range(B):
        lead = b - b % groups
        lens[b] = lens[lead] if groups > 1 else lens[b]
        k, shared = -(-lens[b] // page), lens[b] // page // 2 if b != lead else 0
        tables[b, :shared] = tables[lead, :shared]
        tables[b, shared:k] = order[at:at + k - shared]
        at += k - shared
    return rng, tables.astype(np.int32), lens.astype(np.int32)


def _check_step(got, before, want, lens):
    if want is None:
        assert got["status"][0] != 0
        return
    assert got["status"][0] == 0
    for k in ("lens", "slots", "positions", "copies"):
        assert got[k].tolist() == want[k], k
    assert got["cu"].tolist() == want["cu_new"]
    for b, row in enumerate(want["rows"]):
        assert got["tables"][b, :len(row)].tolist() == row, b
        assert np.array_equal(got["tables"][b, len(row):], before[b, len(row):])


@pytest.mark.parametrize("B,page,longest,n_pages,groups,new", [
    (1, 16, 0, 1, 1, 1), (1, 1, 40, 64, 1, 3), (3, 16, 100, 33, 1, 1), (8, 24, 1000, 700, 4, 1), (33, 16, 300, 2000, 1, 40),
    (64, 8, 500, 6000, 8, 1), (255, 32, 900, 9000, 5, 2), (1100, 16, 60, 8000, 1, 1), (4096, 4, 30, 40000, 2, 1), (2, 16, 40000, 6000, 2, 700)])
@pytest.mark.parametrize("mode", ["go on", "in place", "beams", "come and go"])
def test_step(kq, B, page, longest, n_pages, groups, new, mode):
    width = -(-(longest + new) // page) + 1
    rng, tables, lens = _state(B + page, B, page, longest, n_pages, width, groups if mode in ("beams", "go on") else 1)
    held = (rng.random(n_pages) < 0.02).astype(np.uint8) if n_pages > 100 else None
    more = rng.integers(0, new + 1, B) if new > 1 else np.full(B, new)
    parents = None
    if mode == "beams":
        parents = np.arange(B) // groups * groups + rng.integers(0, groups, B)
        parents = np.minimum(parents, B - 1)
    if mode == "come and go":
        parents = np.where(rng.random(B) < 0.3, -1, rng.permutation(B))
    max_new = int(more.sum()) + 5
    s = Step(kq, tables, lens, parents, more, held, n_pages, page, max_new, mode == "in place")
    before = tables.copy() if mode == "in place" else np.full(tables.shape, -77)
    got = s.run()
    _check_step(got, before, pr.step(tables, lens, parents, more, held, n_pages, page, max_new), lens)


@pytest.mark.parametrize("seed", range(24))
def test_steps_of_any_shape(kq, seed):
    """Random shapes, parents from anywhere in the batch, some steps that cannot take place."""
    rng = np.random.default_rng(1000 + seed)
    B, page = int(rng.integers(1, 200)), int(rng.choice([1, 3, 8, 16, 31, 64, 257]))
    longest = int(rng.integers(0, 40 * page))
    width = longest // page + 3
    n_pages = int(B * (longest / page + 1) * 1.2 + 4)
    _, tables, lens = _state(seed, B, page, longest, n_pages, width)
    parents = rng.integers(-1, B, B)
    new = rng.integers(0, 2 * page + 1, B)
    max_new = int(new.sum() * rng.choice([0.9, 1.0, 1.5])) + 1
    s = Step(kq, tables, lens, parents, new, None, n_pages, page, max_new)
    got, want = s.run(), pr.step(tables, lens, parents, new, None, n_pages, page, max_new)
    if want is not None:
        before = np.full(tables.shape, -77)
    else:
        before = None
    _check_step(got, before, want, lens)
    if want is None:
        _unchanged(got, tables, lens, page)


def _unchanged(got, tables, lens, page):
    assert got["lens"].tolist() == lens.tolist()
    for b, n in enumerate(lens):
        k = -(-max(int(n), 0) // page)
        if k <= tables.shape[1]:
            assert np.array_equal(got["tables"][b, :k], tables[b, :k])
    assert not got["cu"].any() and np.all(got["slots"] == -1) and np.all(got["positions"] == -1)
    assert np.array_equal(got["copies"], np.tile([-1, -1, 0], (len(lens), 1)))


def test_steps_that_do_not_take_place(kq):
    page, width, n_pages = 8, 6, 40
    _, tables, lens = _state(3, 5, page, 24, n_pages, width)
    lens[:] = [20, 3, 0, 8, 17]
    order = iter(range(n_pages))
    for b in range(5):
        for j in range(-(-lens[b] // page)):
            tables[b, j] = next(order)
    keep, one = list(range(5)), [1] * 5

    def status(t=tables, n=lens, p=keep, new=one, held=None, pages=n_pages, room=64):
        s = Step(kq, t, n, p, new, held, pages, page, room)
        got = s.run()
        if got["status"][0]:
            _unchanged(got, t, np.asarray(n), page)
        return int(got["status"][0])

    used = sum(-(-n // page) for n in lens)            # 8 pages; rows 2 and 3 want one more each
    assert status(pages=used + 2) == 0 and status(pages=used + 1) == kq.KVQ_PAGE_FULL
    assert status(held=[0] * used + [1] * (n_pages - used)) == kq.KVQ_PAGE_FULL
    assert status(new=[28, 1, 1, 1, 1]) == 0 and status(new=[29, 1, 1, 1, 1]) == kq.KVQ_PAGE_LONG
    assert status(new=[2 ** 31 - 1] * 5) & kq.KVQ_PAGE_LONG
    assert status(room=5) == 0 and status(room=4) == kq.KVQ_PAGE_SLOTS and status(room=0) == kq.KVQ_PAGE_SLOTS
    assert status(new=[0] * 5, room=0) == 0
    for bad in ([0, 1, 2, 3, 5], [0, 1, -2, 3, 4], [0, 2 ** 30, 2, 3, 4]):
        assert status(p=bad) == kq.KVQ_PAGE_BAD
    assert status(new=[1, -1, 1, 1, 1]) == kq.KVQ_PAGE_BAD
    assert status(n=np.array([-1, 3, 0, 8, 17], np.int32)) == kq.KVQ_PAGE_BAD
    assert status(n=np.array([49, 3, 0, 8, 17], np.int32)) & kq.KVQ_PAGE_BAD
    assert status(n=np.array([49, 3, 0, 8, 17], np.int32), p=[1, 1, 2, 3, 4]) == 0      # nobody takes that row
    for page_number in (-1, n_pages, 2 ** 31 - 1):
        t = tables.copy()
        t[0, 1] = page_number
        assert status(t=t) == kq.KVQ_PAGE_BAD
        t = tables.copy()
        t[4, 2] = page_number                          # the partly filled one, that only a copy would read
        assert status(t=t, p=[4, 4, 2, 3, 3]) == kq.KVQ_PAGE_BAD
    assert status(p=[-1] * 5, new=[0] * 5, pages=1) == 0


def test_step_of_an_empty_batch(kq):
    import torch
    i32 = lambda n: torch.full((n,), -77, dtype=torch.int32, device="cuda")
    cu, status, pos, slots = i32(1), i32(1), i32(3), torch.full((3,), -77, dtype=torch.int64, device="cuda")
    kq.kvq_page_step(None, None, 4, None, None, None, None, 0, None, 10, 16, 3, cu, slots, pos, None, status)
    assert cu.item() == 0 and status.item() == 0 and slots.tolist() == [-1] * 3 and pos.tolist() == [-1] * 3


def test_step_with_the_most_pages_and_rows(kq):
    B, n_pages = 4096, 1 << 20
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 3, B).astype(np.int32)
    order = rng.permutation(n_pages)
    tables = np.full((B, 4), -1, np.int32)
    tables[:, 0], tables[:, 1] = order[:B], order[B:2 * B]
    held = np.ones(n_pages, np.uint8)
    held[-2 * B:] = 0                                  # what is free lies at the end
    got = Step(kq, tables, lens, np.arange(B), [1] * B, held, n_pages, 1, B).run()
    _check_step(got, np.full(tables.shape, -77), pr.step(tables, lens, None, [1] * B, held, n_pages, 1, B), lens)


# ---------------------------------------------------------------- rows by slot

def _cache_tensors(n_pages, page, H, D, dtype, order="slots", fill=float("nan")):
    import torch
    if order == "slots":
        return [torch.full((n_pages, page, H, D), fill, dtype=dtype, device="cuda") for _ in range(2)]
    if order == "heads":
        return [torch.full((n_pages, H, page, D), fill, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2)]
    both = torch.full((n_pages, 2, page, H + 1, D + 8), fill, dtype=dtype, device="cuda")      # keys and values together, with gaps
    return [both[:, i, :, :H, :D] for i in range(2)]


@pytest.mark.parametrize("order", ["slots", "heads", "together"])
@pytest.mark.parametrize("n,H,D,page,copies", [(1, 1, 8, 1, 0), (7, 3, 64, 16, 3), (100, 5, 64, 24, 9), (33, 2, 128, 8, 1), (5, 32, 128, 64, 0), (600, 7, 72, 5, 20),
                                               (3, 100, 128, 4, 2), (0, 3, 64, 16, 4)])
def test_append(kq, n, H, D, page, copies, order):
    import torch
    rng = np.random.default_rng(n + H)
    n_pages = n // page + 2 * copies + 4
    dtype = torch.bfloat16 if n % 2 else torch.float16
    g = torch.Generator(device="cuda").manual_seed(n)
    K, V = _cache_tensors(n_pages, page, H, D, dtype, order)
    for c in (K, V):
        c.copy_(torch.randn(c.shape, generator=g, device="cuda"))
    want = [c.clone() for c in (K, V)]
    rows = [torch.randn((n, H, D), generator=g, device="cuda").to(dtype) for _ in range(2)]
    pages = rng.permutation(n_pages)
    pool = (pages[2 * copies:, None] * page + np.arange(page)).ravel()
    slots = rng.permutation(pool)[:n].astype(np.int64)
    slots[rng.random(n) < 0.2] = -1
    if n > 3:
        slots[-2:] = [n_pages * page, 2 ** 62]         # outside the cache
    cp = np.stack([pages[:copies], pages[copies:2 * copies], rng.integers(1, page + 1, copies)], 1).astype(np.int32)
    if copies > 3:
        cp[1], cp[2], cp[3] = [-1, -1, 0], [cp[2][0], n_pages, 2], [n_pages, cp[3][1], 1]
    for i, (w, r) in enumerate(zip(want, rows)):
        for s, d, k in cp.tolist():
            if 0 <= s < n_pages and 0 <= d < n_pages:
                w[d, :k] = w[s, :k]
        for t, s in enumerate(slots.tolist()):
            if 0 <= s < n_pages * page:
                w[s // page, s % page] = r[t]
    whole = K.untyped_storage() if order == "together" else None
    gaps = None if whole is None else torch.as_strided(K, (n_pages, 2, page, H + 1, D + 8), (2 * page * (H + 1) * (D + 8), page * (H + 1) * (D + 8), (H + 1) * (D + 8), D + 8, 1))
    kq.kvq_page_append(kq.kvq_page_cache(K, V), *rows, torch.from_numpy(slots).cuda(), n, torch.from_numpy(cp).cuda() if copies else None, copies)
    torch.cuda.synchronize()
    assert torch.equal(K, want[0]) and torch.equal(V, want[1])
    if gaps is not None:
        assert torch.isnan(gaps[:, :, :, H:]).all() and torch.isnan(gaps[:, :, :, :, D:]).all()


# ---------------------------------------------------------------- attention

class Attn:
    """A cache of random rows (everything else NaN) and one call's buffers."""

    def __init__(self, kq, lens, q_heads, kv_heads, D, page, dtype="fp16", order="slots", seed=0, sharp=1.0, width=None, bad=0.0):
        import torch
        self.kq, self.lens, self.Hq, self.H, self.D, self.page = kq, [int(n) for n in lens], q_heads, kv_heads, D, page
        self.dtype = torch.float16 if dtype == "fp16" else torch.bfloat16
        self.mantissa = 11 if dtype == "fp16" else 8
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        pages = [-(-n // page) for n in self.lens]
        n_pages = sum(pages) + 3
        self.width = width or max(1, max(pages))
        self.K, self.V = _cache_tensors(n_pages, page, kv_heads, D, self.dtype, order)
        perm, at = rng.permutation(n_pages), 0
        tables = rng.integers(-2, 2 ** 31 - 1, (len(lens), self.width)).astype(np.int32)
        self.rows, self.live = [], []
        for b, (n, k) in enumerate(zip(self.lens, pages)):
            tables[b, :k] = perm[at:at + k]
            at += k
            where = torch.from_numpy(tables[b, :k].astype(np.int64)).cuda()
            pair = []
            for c, f in ((self.K, sharp), (self.V, 1.0)):
                x = (torch.randn((k * page, kv_heads, D), generator=g, device="cuda") * f).to(self.dtype)
                x[n:] = float("nan")
                c[where] = x.reshape(k, page, kv_heads, D)
                pair.append(x[:n].double().cpu().numpy())
            live = np.ones(n, bool)
            for j in range(k):                         # pages that are not there
                if rng.random() < bad:
                    tables[b, j] = rng.choice([-1, n_pages, 2 ** 31 - 1])
                    live[j * page:(j + 1) * page] = False
            self.rows.append(pair)
            self.live.append(live)
        self.Q = torch.randn((len(lens), q_heads, D), generator=g, device="cuda").to(self.dtype)
        self.tables = torch.from_numpy(tables).cuda()
        self.n = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.cache = kq.kvq_page_cache(self.K, self.V)
        self.O = torch.full_like(self.Q, float("nan"))
        self.lse = torch.full((len(lens), q_heads), float("nan"), device="cuda")
        self.scale = D ** -0.5
        self.bytes = kq.kvq_page_attn_workspace_bytes(len(lens), q_heads, kv_heads, D)
        self.work = torch.zeros(self.bytes, dtype=torch.uint8, device="cuda")

    def call(self, lse=True):
        self.kq.kvq_page_attn(self.cache, self.Q, self.O, self.lse if lse else None, self.tables, self.width, self.n, len(self.lens), self.Hq,
                              self.scale, self.work, self.bytes)

    def check(self, heads=None, pairs=None):
        """Every (row, KV head), those of some heads, or only some pairs."""
        import torch
        torch.cuda.synchronize()
        O, lse, Q = self.O.double().cpu().numpy(), self.lse.double().cpu().numpy(), self.Q.double().cpu().numpy()
        G, worst = self.Hq // self.H, 0.0
        for b, (k, v) in enumerate(self.rows):
            k, v = k[self.live[b]], v[self.live[b]]
            for h in [h for h in (heads or range(self.H)) if pairs is None or (b, h) in pairs]:
                at = slice(h * G, h * G + G)
                o, l, err, lerr = pr.attend(Q[b, at], k[:, h], v[:, h], self.scale, self.mantissa)
                assert np.all(np.isfinite(O[b, at])), (b, h)
                over = np.abs(O[b, at] - o) / np.maximum(err, 1e-300)
                assert np.all(np.abs(O[b, at] - o) <= err), (b, h, over.max())
                if len(k):
                    assert np.all(np.abs(lse[b, at] - l) <= lerr), (b, h)
                    worst = max(worst, over.max())
                else:
                    assert np.all(lse[b, at] == -math.inf) and not O[b, at].any()
        assert not self.work[:8192].any()              # the counters are back at zero
        return worst


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (9, 3), (8, 1), (9, 1), (32, 2), (21, 1), (15, 5), (12, 12)])
def test_attention_of_short_and_odd_lengths(kq, q_heads, kv_heads, D, dtype):
    a = Attn(kq, [0, 1, 2, 15, 16, 17, 31, 33, 0, 0, 64, 100, 127, 1, 300], q_heads, kv_heads, D, 16, dtype)
    a.call()
    a.check()


@pytest.mark.parametrize("order", ["slots", "heads", "together"])
@pytest.mark.parametrize("page", [1, 3, 8, 24, 64, 100, 1024])
def test_attention_over_pages_of_any_size_and_order(kq, page, order):
    for D, dtype in ((64, "bf16"), (128, "fp16")):
        a = Attn(kq, [37, 1, 500, 0, 1023, 1], 6, 2, D, page, dtype, order, seed=page)
        a.call()
        a.check()


@pytest.mark.parametrize("lens,q_heads,kv_heads,D", [
    ([20000], 3, 1, 64), ([30011], 15, 5, 64), ([9999, 3], 8, 8, 128), ([4097] * 5, 32, 8, 128), ([700] * 64, 9, 3, 64), ([50, 6000, 7, 1, 3000] * 9, 4, 4, 64),
    ([5] * 700, 8, 8, 64), ([17, 0] * 900, 2, 1, 128), ([2048] * 16, 32, 32, 64)])
def test_attention_split_over_many_warps(kq, lens, q_heads, kv_heads, D):
    a = Attn(kq, lens, q_heads, kv_heads, D, 16, "fp16", seed=len(lens))
    a.call()
    a.check(heads=range(min(kv_heads, 3)))


@pytest.mark.parametrize("lens,q_heads,kv_heads,D", [
    ([65536], 8, 2, 64), ([70000, 3, 20000], 9, 3, 64), ([40000], 2, 2, 128), ([40000, 500, 0, 9000], 16, 1, 128), ([50000], 20, 1, 64),
    ([20000, 100, 5000] * 8, 6, 2, 64), ([16000, 40] * 35, 4, 2, 64), ([9000, 33, 1] * 24, 2, 1, 128), ([31000, 17, 0] * 3, 33, 1, 128)])
def test_attention_of_units_longer_than_equal_shares(kq, lens, q_heads, kv_heads, D):
    """Clusters that share units with one another."""
    a = Attn(kq, lens, q_heads, kv_heads, D, 16, "bf16", seed=len(lens))
    for _ in range(2):
        a.call()
    a.check()


@pytest.mark.parametrize("q_heads,kv_heads,D,rows", [(42, 2, 64, 90), (33, 1, 64, 100), (64, 2, 128, 90), (10, 10, 64, 40), (6, 6, 64, 33)])
@pytest.mark.parametrize("order", ["slots", "heads"])
def test_attention_of_many_rows_and_heads_side_by_side(kq, q_heads, kv_heads, D, rows, order):
    """Equal shares of the work, of one unit at a time and of two, with borders inside units and moved ones."""
    rng = np.random.default_rng(rows)
    lens = np.where(rng.random(rows) < 0.2, 0, rng.integers(1, 1500, rows))
    a = Attn(kq, lens, q_heads, kv_heads, D, 16, "fp16", order, seed=rows)
    a.call()
    a.check(pairs={(b, h) for b in range(0, rows, 3) for h in range(kv_heads)})


@pytest.mark.parametrize("seed", range(40))
def test_attention_of_any_shape(kq, seed):
    rng = np.random.default_rng(seed)
    kv, group, D = int(rng.choice([1, 2, 3, 4, 5, 8, 12])), int(rng.choice([1, 2, 3, 7, 8, 9, 16, 17, 33])), int(rng.choice([64, 64, 128]))
    rows, top = int(np.exp(rng.uniform(0, np.log(300)))), int(np.exp(rng.uniform(0, np.log(20000))))
    while rows * kv * top * D > 5e7:
        rows, top = max(1, rows // 2), top if rows > 1 else top // 2
    kind = rng.integers(3)
    lens = [rng.integers(0, top + 1, rows), np.full(rows, top), np.where(rng.random(rows) < 0.1, top, rng.integers(0, max(2, top // 20), rows))][kind]
    page = int(rng.choice([1, 5, 8, 16, 24, 64, 200]))
    a = Attn(kq, lens, kv * group, kv, D, page, str(rng.choice(["fp16", "bf16"])), str(rng.choice(["slots", "heads", "together"])), seed=seed,
             width=max(1, -(-int(max(lens)) // page)) * int(rng.choice([1, 1, 4])), bad=float(rng.choice([0, 0, 0.1])))
    a.call()
    a.call()                                           # (the workspace is as good as new)
    a.check(pairs={(int(b), int(rng.integers(kv))) for b in [*rng.integers(0, rows, 6), 0, rows - 1, int(np.argmax(lens))]})


@pytest.mark.parametrize("lens,q_heads,kv_heads", [([700], 9, 3), ([30000], 9, 3), ([900, 0, 77, 4000] * 6, 32, 8)])
def test_attention_writes_over_its_queries(kq, lens, q_heads, kv_heads):
    a = Attn(kq, lens, q_heads, kv_heads, 64, 16)
    a.call()
    want, a.O = a.O.clone(), a.Q
    a.call()
    assert want.equal(a.O)


@pytest.mark.parametrize("rows,q_heads,kv_heads", [(4096, 4, 2), (2200, 3, 3), (2047, 12, 1)])
def test_attention_of_very_many_rows(kq, rows, q_heads, kv_heads):
    rng = np.random.default_rng(rows)
    lens = rng.integers(0, 60, rows)
    lens[[0, 7, rows // 2, rows - 1]] = 9000, 3, 17000, 1
    a = Attn(kq, lens, q_heads, kv_heads, 64, 32)
    a.call()
    a.check()


def test_attention_of_the_largest_batch(kq):
    rng = np.random.default_rng(5)
    a = Attn(kq, rng.integers(0, 40, 4096), 2, 2, 128, 8, "bf16")
    a.call()
    a.check()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("sharp", [0.0, 8.0, 60.0])
def test_attention_flat_and_peaked(kq, sharp, dtype):
    a = Attn(kq, [3000, 1500, 40], 6, 2, 64, 16, dtype, sharp=sharp)
    a.call()
    a.check()


def test_attention_with_rising_logits(kq):
    """Every tile has a new maximum: the reference moves at each of them."""
    import torch
    a = Attn(kq, [2000], 3, 1, 64, 16, "fp16")
    ramp = torch.linspace(-1, 1, 2000, device="cuda")
    flat = a.tables[0, :125].long()
    a.K[flat] = (ramp[:, None, None] * 30 * torch.ones(64, device="cuda")).half().reshape(125, 16, 1, 64)
    a.Q[:] = 1.0
    a.Q[0, 1] = -1.0
    a.rows[0][0] = a.K[flat].reshape(2000, 1, 64).double().cpu().numpy()
    a.call()
    a.check()


def test_attention_scales_and_missing_outputs(kq):
    import torch
    for scale in (0.0, -0.1, 1.0):
        a = Attn(kq, [100, 5], 4, 2, 64, 16)
        a.scale = scale
        a.call()
        a.check()
        want = a.O.clone()
        a.O.fill_(float("nan"))
        a.lse.fill_(7.0)
        a.call(lse=False)
        torch.cuda.synchronize()
        assert torch.equal(a.O, want) and torch.all(a.lse == 7.0)


@pytest.mark.parametrize("page", [3, 16, 40])
def test_attention_with_pages_that_are_not_there(kq, page):
    a = Attn(kq, [900, 50, 16, 17, 5], 6, 2, 64, page, "bf16", bad=0.4, seed=page)
    a.call()
    a.check()
    b = Attn(kq, [900, 50], 6, 2, 64, page, "fp16", bad=1.0)
    b.call()
    b.check()


def test_attention_with_lengths_out_of_range(kq):
    import torch
    a = Attn(kq, [64, 20, 48], 6, 2, 64, 16, width=4)
    a.n = torch.tensor([2 ** 31 - 1, -5, 48], dtype=torch.int32, device="cuda")       # the table's width counts; nothing
    a.lens[1], a.rows[1], a.live[1] = 0, [r[:0] for r in a.rows[1]], a.live[1][:0]
    a.call()
    a.check()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_attention_passes_on_what_is_not_finite(kq, dtype):
    import torch
    a = Attn(kq, [200, 200, 200], 4, 2, 64, 16, dtype)
    where = lambda b, t: (int(a.tables[b, t // 16]), t % 16)
    a.V[where(0, 77) + (0, 5)] = float("nan")          # a value that is seen: its channel, in the heads that read it
    a.K[where(1, 3) + (1, 9)] = float("nan")           # a key: the whole row
    a.V[where(2, 199) + (1, 63)] = float("inf")
    a.call()
    O = a.O.float().cpu()
    bad = torch.zeros_like(O, dtype=torch.bool)
    bad[0, :2, 5] = bad[1, 2:] = bad[2, 2:, 63] = True
    assert torch.isfinite(O[~bad]).all() and not torch.isfinite(O[bad]).any()


def test_equal_calls_give_equal_bits_and_workspaces_serve_any_shape(kq):
    import torch
    a = Attn(kq, [3000, 17, 900, 5000], 15, 5, 64, 16, "bf16")
    b = Attn(kq, [1, 700], 40, 2, 128, 16)
    size = max(a.bytes, b.bytes)
    a.work = b.work = torch.zeros(size, dtype=torch.uint8, device="cuda")
    a.bytes = b.bytes = size
    first = []
    for i in range(20):
        a.call()
        b.call()
        first.append((a.O.clone(), b.O.clone(), a.lse.clone()))
    torch.cuda.synchronize()
    for x in first:
        assert all(torch.equal(p, q) for p, q in zip(x, first[0]))
    a.check()
    b.check()


def test_attention_does_not_depend_on_where_a_row_lies(kq):
    """The same request in every row of a batch gives the same numbers to the error of the sums."""
    import torch
    a = Attn(kq, [1234], 9, 3, 64, 16)
    a.call()
    want, lse = a.O.double(), a.lse.double()
    for n in (2, 50):
        a.tables = a.tables[:1].repeat(n, 1).contiguous()
        a.n, a.Q, a.lens = a.n[:1].repeat(n).contiguous(), a.Q[:1].repeat(n, 1, 1).contiguous(), [1234] * n
        a.O, a.lse = torch.empty_like(a.Q), torch.empty((n, 9), device="cuda")
        a.call()
        assert (a.O.double() - want).abs().max() <= 2.0 ** -10 * want.abs().max() and (a.lse.double() - lse).abs().max() < 1e-5


def test_attention_in_a_graph_follows_lengths_and_tables(kq):
    import torch
    a = Attn(kq, [500, 3, 900], 6, 2, 64, 16, width=64)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a.call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.call()
    b = Attn(kq, [40, 0, 1000], 6, 2, 64, 16, width=64, seed=9)
    k = b.K.shape[0]                                   # (the second cache fits the first)
    a.K[:k], a.V[:k] = b.K, b.V
    a.tables.copy_(b.tables)
    a.n.copy_(b.n)
    a.Q.copy_(b.Q)
    a.rows, a.live, a.lens = b.rows, b.live, b.lens
    for _ in range(3):
        a.O.fill_(float("nan"))
        graph.replay()
        a.check()


def test_attention_of_a_cache_whose_offsets_pass_32_bits(kq):
    import torch
    far = 2 ** 30 + 64                                 # elements between pages: the last starts 6.4 GB into the cache
    try:
        both = torch.empty(3 * far + 4 * 16 * 2 * 64, dtype=torch.float16, device="cuda")
    except torch.cuda.OutOfMemoryError:
        pytest.skip("needs 6.5 GB")
    K = torch.as_strided(both, (4, 16, 2, 64), (far, 128, 64, 1), 0)
    V = torch.as_strided(both, (4, 16, 2, 64), (far, 128, 64, 1), 16 * 2 * 64)
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = [torch.randn((60, 2, 64), generator=g, device="cuda").half() for _ in range(2)]
    tables = torch.tensor([[3, 0, 2, 1]], dtype=torch.int32, device="cuda")
    t = torch.arange(60, device="cuda")
    slots = tables[0, t // 16].long() * 16 + t % 16
    cache = kq.kvq_page_cache(K, V)
    kq.kvq_page_append(cache, *rows, slots, 60)
    assert torch.equal(K[tables[0].long()].reshape(64, 2, 64)[:60], rows[0]) and torch.equal(V[tables[0].long()].reshape(64, 2, 64)[:60], rows[1])
    a = Attn(kq, [60], 6, 2, 64, 16)
    a.K, a.V, a.cache, a.tables, a.width = K, V, cache, tables, 4
    a.rows = [[r.double().cpu().numpy() for r in rows]]
    a.call()
    a.check()


def test_requests_that_come_share_grow_and_go(kq):
    """Tables, appended rows and attention together, over 40 steps with forks, against rows kept on the host."""
    import torch
    rng = np.random.default_rng(11)
    B, H, Hq, D, page, n_pages, width = 6, 2, 6, 64, 8, 90, 24
    K, V = _cache_tensors(n_pages, page, H, D, torch.float16)
    cache = kq.kvq_page_cache(K, V)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    tables, lens = [i32(B, width), i32(B, width)], i32(B)
    cu, copies, status = i32(B + 1), i32(B, 3), i32(1)
    slots, positions = torch.zeros(64, dtype=torch.int64, device="cuda"), i32(64)
    kept = [(np.zeros((0, H, D)), np.zeros((0, H, D))) for _ in range(B)]
    size = kq.kvq_page_attn_workspace_bytes(B, Hq, H, D)
    work = torch.zeros(size, dtype=torch.uint8, device="cuda")
    took_place = 0
    for step in range(40):
        new = rng.integers(0, 3, B)
        parents = np.arange(B)
        if step % 3 == 0:
            parents = rng.integers(0, B, B)            # forks anywhere
        if step % 5 == 0:
            parents[rng.integers(0, B)] = -1           # a request leaves, another comes with its prompt
        new = np.where(parents < 0, rng.integers(1, 10, B), new)
        total = int(new.sum())
        src, dst = tables[step % 2], tables[(step + 1) % 2]
        kq.kvq_page_step(src, dst, width, lens, lens, torch.tensor(parents, dtype=torch.int32).cuda(), torch.tensor(new, dtype=torch.int32).cuda(), B,
                         None, n_pages, page, 64, cu, slots, positions, copies, status)
        rows = [torch.randn((64, H, D), device="cuda").half() for _ in range(2)]
        kq.kvq_page_append(cache, *rows, slots, 64, copies, B)
        if status.item() == 0:
            took_place += 1
            old, kept, at = kept, [], 0
            for b in range(B):
                k, v = old[parents[b]] if parents[b] >= 0 else (np.zeros((0, H, D)), np.zeros((0, H, D)))
                mine = [r[at:at + new[b]].double().cpu().numpy() for r in rows]
                kept.append((np.concatenate([k, mine[0]]), np.concatenate([v, mine[1]])))
                at += new[b]
            assert at == total
        assert lens.tolist() == [len(k) for k, _ in kept]
        Q, O = torch.randn((B, Hq, D), device="cuda").half(), torch.zeros((B, Hq, D), dtype=torch.float16, device="cuda")
        kq.kvq_page_attn(cache, Q, O, None, dst, width, lens, B, Hq, D ** -0.5, work, size)
        q, o = Q.double().cpu().numpy(), O.double().cpu().numpy()
        for b, (k, v) in enumerate(kept):
            for h in range(H):
                want, _, err, _ = pr.attend(q[b, 3 * h:3 * h + 3], k[:, h], v[:, h], D ** -0.5, 11)
                assert np.all(np.abs(o[b, 3 * h:3 * h + 3] - want) <= err), (step, b, h)
    assert took_place >= 20


def test_calls_on_another_stream(kq):
    import torch
    a = Attn(kq, [700, 20], 9, 3, 64, 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.call()
    side.synchronize()
    a.check()
