"""Limits of the paged cache's calls from both sides, nothing of which reaches a GPU."""
import ctypes as C

import pytest

from test_pages_refusals import A, ARG, ATTN, SELECT, STEP, _cache


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


@pytest.mark.parametrize("change,code", [(dict(kv_heads=1024), 0), (dict(kv_heads=1025), ARG), (dict(head_dim=1024), 0), (dict(head_dim=1032), ARG)])
def test_heads_and_channels_of_a_cache(kq, change, code):
    c = _cache(kq, **change)
    assert kq.lib().kvq_page_append(C.byref(c), None, None, None, 0, None, 0, None) == code


@pytest.mark.parametrize("kv_heads,q_heads,code", [(1, 16384, 0), (1, 16385, ARG), (1024, 16384, 0), (1024, 17408, ARG), (1025, 1025, ARG), (3, 16383, 0), (3, 16386, ARG)])
def test_query_heads(kq, kv_heads, q_heads, code):
    c, n = _cache(kq, kv_heads=kv_heads), C.c_uint64()
    assert kq.lib().kvq_page_attn(C.byref(c), *dict(ATTN, q_heads=q_heads, batch=0).values(), None) == code
    if code:
        assert kq.lib().kvq_page_attn_workspace_bytes(1, q_heads, kv_heads, 64, C.byref(n)) == code


def test_rows_of_a_batch(kq):
    c = _cache(kq)
    assert kq.lib().kvq_page_append(C.byref(c), None, None, None, 0, None, 1 << 30, None) == 0          # (without copies nothing has a batch)
    wide = _cache(kq, kv_heads=128)                    # (a block for every token)
    assert kq.lib().kvq_page_append(C.byref(wide), A, A, A, 2 ** 31 - 4096, A, 4096, None) == ARG        # n_new + batch = 2^31
    assert kq.lib().kvq_page_step(*dict(STEP, batch=4097).values(), None) == ARG
    assert kq.lib().kvq_beam_select(*dict(SELECT, batch=(1 << 24) + 1).values(), None) == ARG
