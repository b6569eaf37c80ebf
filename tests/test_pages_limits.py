"""Limits of the paged cache's calls from both sides, nothing of which reaches a GPU."""
import ctypes as C

import pytest

from test_pages_refusals import A, ARG, ATTN, _cache


@pytest.fixture(scope="module")
def kq():
    from paper_2604_04722_b200 import binding, build
    build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("scale,code", [(2e38, 0), (-2e38, 0), (2.4e38, ARG), (-2.4e38, ARG), (3.4e38, ARG), (1e-45, 0), (0.0, 0)])
def test_scales_that_overflow_in_log2_units(kq, scale, code):
    c = _cache(kq)
    assert kq.lib().kvq_page_attn(C.byref(c), *dict(ATTN, scale=scale, batch=0).values(), None) == code
