"""The paged attention where single numbers go wrong, such as logits of great size (GPU)."""
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
