"""The paged attention where single numbers go wrong: weights far below the largest, logits and values of great size, keys and values
that are not finite, what is left in the workspace (GPU)."""
import math

import numpy as np
import pytest

import pages_reference as pr
from test_gpu_pages import Attn

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


def _sink(kq, rows, n, q_heads, kv_heads, D, dtype, order, gap, spread, sink_value, mean, seed=0):
    """`rows` requests over the same pages: token 0 has the logit 0 and small values, the others lie `gap` and up to `spread` below it."""
    import torch
    rng = np.random.default_rng(seed)
    a = Attn(kq, [n], q_heads, kv_heads, D, 16, dtype, order, seed=seed)
    k, v = np.zeros((n, kv_heads, D)), rng.standard_normal((n, kv_heads, D)) + mean
    k[1:, :, 0] = -gap - spread * rng.random((n - 1, kv_heads))
    v[0] = sink_value
    where = a.tables[0, :n // 16].long()
    for c, x in ((a.K, k), (a.V, v)):
        c[where] = torch.tensor(x, device="cuda").to(a.dtype).reshape(n // 16, 16, kv_heads, D)
    a.rows = [[c[where].reshape(n, kv_heads, D).double().cpu().numpy() for c in (a.K, a.V)]]
    a.Q = torch.zeros((rows, q_heads, D), dtype=a.dtype, device="cuda")
    a.Q[:, :, 0] = D ** 0.5                            # (16-bit for 64 channels; near enough for 128)
    a.scale = 1.0 / float(a.Q[0, 0, 0])
    a.tables, a.n = a.tables.repeat(rows, 1).contiguous(), a.n.repeat(rows).contiguous()
    a.O, a.lse = torch.full_like(a.Q, float("nan")), torch.full((rows, q_heads), float("nan"), device="cuda")
    a.lens = [n] * rows
    return a


def _bound(q, k, v, scale, mantissa):
    """pr.attend's, but with what two fp16 numbers of a weight really leave: the weights are 2^7 and more at the largest, the second number
    holds 2^11 times what the first left, so that a weight is cut at 2^-25 2^-11 2^-7 of the largest; and the values that the second
    is multiplied with, 2^-11 times their size, are cut at 2^-25, which at most half of the weight, or 2^-46 of the largest, sees."""
    o, lse, err, lerr = pr.attend(q, k, v, scale, mantissa)
    if mantissa == 11:
        z = (q @ k.T) * scale
        total = np.exp(z - z.max(1, keepdims=True)).sum(1, keepdims=True)
        err = err + (2.0 ** -43 - 2.0 ** -25) * np.abs(v).sum(0) / total + 2.0 ** -26 + len(k) * 2.0 ** -46 / total
    return o, lse, err, lerr


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("q_heads,kv_heads,D,rows,n", [(3, 3, 64, 1024, 8192), (4, 2, 64, 1200, 4096), (9, 1, 64, 2200, 4096), (2, 2, 128, 700, 8192),
                                                       (12, 1, 128, 1300, 2048), (1, 1, 64, 1, 65536), (2, 1, 64, 4096, 512)])
@pytest.mark.parametrize("gap,spread,sink_value,mean", [(16.0, 0.0, 0.0, 1.0), (17.25, 0.0, 0.0, 1.0), (17.5, 0.0, 0.0, 1.0), (19.0, 0.0, 0.0, 2.0), (14.0, 2.0, 0.0, 0.0),
                                                       (10.0, 8.0, 0.01, 0.0), (16.0, 4.0, 0.0, 0.5)])
def test_attention_next_to_a_token_that_takes_nearly_all_of_the_weight(kq, gap, spread, sink_value, mean, q_heads, kv_heads, D, rows, n, dtype):
    """The sum of what the others have decides the output although each of their weights is below 2^-20 of the largest."""
    import torch
    a = _sink(kq, rows, n, q_heads, kv_heads, D, dtype, "slots", gap, spread, sink_value, mean)
    a.call()
    torch.cuda.synchronize()
    O, lse, G = a.O.double().cpu().numpy(), a.lse.double().cpu().numpy(), q_heads // kv_heads
    q = a.Q[0].double().cpu().numpy()
    for h in range(kv_heads):
        at = slice(h * G, h * G + G)
        o, l, err, lerr = _bound(q[at], a.rows[0][0][:, h], a.rows[0][1][:, h], a.scale, a.mantissa)
        over = np.abs(O[:, at] - o) / err
        assert np.all(over <= 1), (h, over.max())
        assert np.all(np.abs(lse[:, at] - l) <= lerr)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [25, 26, 27, 28, 29])
def test_attention_with_logits_whose_steps_are_as_large_as_the_slack(kq, power, D, dtype):
    """Logits of about 2^power in log2 units: neighbouring fp32 numbers are 2 to 64 apart there."""
    import torch
    n = 16 * 40
    a = Attn(kq, [n] * 6, 4, 2, D, 16, dtype, seed=power)
    q, where = torch.zeros_like(a.Q), a.tables.long()
    q[..., 0], q[..., 1] = 1.0, 2.0 ** -7              # products 1024 + j 2^-13: neighbours in fp32
    a.Q = q
    k = torch.zeros((6, n, 2, D), device="cuda")
    k[..., 0] = 1024.0
    k[..., 1] = torch.randint(0, 120, (6, n, 2), device="cuda", generator=torch.Generator(device="cuda").manual_seed(power)) * 2.0 ** -6
    v = torch.rand((6, n, 2, D), device="cuda") + 1.0
    a.K[where], a.V[where] = (x.to(a.dtype).reshape(6, n // 16, 16, 2, D) for x in (k, v))
    a.scale = 1.01 * 2.0 ** (power - 10) / math.log2(math.e)
    a.call()
    torch.cuda.synchronize()
    O = a.O.float()
    assert torch.isfinite(a.lse).all() and torch.isfinite(O).all() and O.min() >= 1.0 and O.max() <= 2.0


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[200, 200, 200], [200, 16, 9000], [1, 1, 1]])
def test_attention_of_infinite_keys_and_values(kq, lens, D, dtype):
    """By the sign of a query's channel a key of +-Inf gives its heads a logit of +Inf (NaN) or -Inf (a weight of zero)."""
    import torch
    a = Attn(kq, lens, 6, 2, D, 16, dtype, seed=D)
    a.Q[:, :, 7] = torch.tensor([1.0, -1.0, 2.0, 1.0, 1.0, -3.0], device="cuda")        # heads 0 to 2 read KV head 0, 3 to 5 the other
    at = lambda b, t: (int(a.tables[b, t // 16]), t % 16)
    last = [n - 1 for n in lens]
    a.K[at(0, last[0]) + (0, 7)] = math.inf
    a.K[at(1, last[1]) + (1, 7)] = -math.inf
    a.V[at(2, last[2]) + (0, 3)] = math.inf
    a.V[at(2, last[2]) + (0, 5)] = -math.inf
    a.call()
    torch.cuda.synchronize()
    O, lse = a.O.double().cpu().numpy(), a.lse.double().cpu().numpy()
    gone = {(0, 0): False, (0, 1): True, (0, 2): False, (1, 3): True, (1, 4): True, (1, 5): False}          # True: without that token
    for b, n in enumerate(lens):
        k, v = a.rows[b]
        for h in range(6):
            g = h // 3
            if gone.get((b, h)) is False:
                assert np.all(np.isnan(O[b, h])) and math.isnan(lse[b, h]), (b, h)
                continue
            kk, vv = (x[:-1, g] if (b, h) in gone else x[:, g] for x in (k, v))
            o, l, err, lerr = pr.attend(a.Q[b, h:h + 1].double().cpu().numpy(), kk, vv, a.scale, a.mantissa)
            some = np.ones(D, bool)
            if b == 2 and g == 0:
                some[[3, 5]] = False
                assert not np.isfinite(O[b, h, [3, 5]]).any()
            assert np.all(np.abs(O[b, h, some] - o[0, some]) <= err[0, some]), (b, h)
            assert lse[b, h] == l[0] or abs(lse[b, h] - l[0]) <= lerr[0]


def test_what_a_call_leaves_in_its_workspace(kq):
    """The arrival counters, 4096 bytes, are back at zero; records behind them may hold anything.  (Units as long as 1.3 warps' shares: CTA 0's
    second warp ends one that the first began and goes on.)"""
    a = Attn(kq, [320] * 600, 3, 3, 64, 16)
    a.work[4096:] = 255
    for _ in range(3):
        a.call()
    o = a.O.clone()
    assert not a.work[:4096].any()
    assert (a.work[6208:6208 + 2112] != 255).any()     # the record of CTA 0's second warp (8 heads of 66 floats)
    a.call()
    assert o.equal(a.O) and o.isfinite().all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[320], [320] * 700, [9000]])
@pytest.mark.parametrize("step", [0.5, 3.0, 5.5, 7.0])
def test_attention_of_very_large_values(kq, step, lens, D):
    """bf16 values near 2^120 under logits that rise from tile to tile: no weight may exceed one, or the sums pass fp32."""
    import torch
    a = Attn(kq, [lens[0]], 4, 2, D, 16, "bf16", seed=D)
    n, where = lens[0], a.tables[0, :-(-lens[0] // 16)].long()
    a.Q = torch.zeros((1, 4, D), dtype=torch.bfloat16, device="cuda")
    a.Q[..., 0], a.scale = 1.0, 1.0
    k = torch.zeros((len(where) * 16, 2, D), device="cuda")
    k[:, :, 0] = (torch.arange(len(k), device="cuda") // 16 % 8)[:, None] * step       # (rises and falls)
    v = (torch.rand(k.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) + 1.0) * 2.0 ** 120
    v[:] *= torch.where(torch.arange(len(k), device="cuda") < 64, 1.0, 2.0 ** -12)[:, None, None]
    for c, x in ((a.K, k), (a.V, v)):
        c[where] = x.bfloat16().reshape(len(where), 16, 2, D)
    a.rows = [[c[where].reshape(-1, 2, D)[:n].double().cpu().numpy() for c in (a.K, a.V)]]
    rows = len(lens)
    a.Q, a.tables, a.n, a.lens = a.Q.repeat(rows, 1, 1), a.tables.repeat(rows, 1).contiguous(), a.n.repeat(rows), lens
    a.O, a.lse = torch.full_like(a.Q, float("nan")), torch.full((rows, 4), float("nan"), device="cuda")
    a.rows, a.live = a.rows * rows, a.live * rows
    a.call()
    a.check(pairs={(b, h) for b in range(0, rows, 50) for h in range(2)})
