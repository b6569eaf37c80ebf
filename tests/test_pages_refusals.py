"""The paged cache and beam search: what the library and the binding refuse before anything is queued, and the plain definitions
that the GPU tests compare with (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest

import pages_reference as pr

ARG, NOMEM = -1, -7
A = 1 << 20                                            # an aligned address that nothing reads


@pytest.fixture(scope="module")
def kq():
    from paper_2604_04722_b200 import binding, build
    build.build()
    binding.lib()
    return binding


STEP = dict(tables_in=A, tables_out=2 * A, width=8, lens_in=A, lens_out=A, parents=None, new_lens=A, batch=4, held=None, n_pages=64,
            page_size=16, max_new=4, cu=A, slots=A, positions=None, copies=None, status=A)


@pytest.mark.parametrize("change", [
    dict(batch=-1), dict(batch=4097), dict(width=0), dict(n_pages=0), dict(n_pages=(1 << 20) + 1), dict(page_size=0), dict(max_new=-1),
    dict(tables_in=None), dict(tables_out=None), dict(lens_in=None), dict(lens_out=None), dict(new_lens=None), dict(cu=None), dict(slots=None),
    dict(status=None), dict(parents=A), dict(parents=A, copies=A, tables_out=A), dict(tables_out=A + 4), dict(lens_out=A + 4),
    dict(tables_in=A + 2), dict(slots=A + 4), dict(copies=A + 1), dict(status=A + 2)])
def test_step_refusals(kq, change):
    assert kq.lib().kvq_page_step(*dict(STEP, **change).values(), None) == ARG


CACHE = dict(K=A, V=2 * A, page_stride=16 * 3 * 64, slot_stride=3 * 64, head_stride=64, n_pages=8, page_size=16, kv_heads=3, head_dim=64, dtype=0)
BAD_CACHES = [dict(K=None), dict(V=None), dict(K=A + 8), dict(V=A + 2), dict(page_stride=4), dict(slot_stride=-64), dict(head_stride=65),
              dict(n_pages=0), dict(n_pages=-1), dict(page_size=0), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=60), dict(dtype=2),
              dict(dtype=-1)]


def _cache(kq, **change):
    return kq.PageCache(*dict(CACHE, **change).values())


@pytest.mark.parametrize("change", BAD_CACHES)
def test_caches_that_are_refused(kq, change):
    c = _cache(kq, **change)
    assert kq.lib().kvq_page_append(C.byref(c), A, A, A, 1, None, 0, None) == ARG
    assert kq.lib().kvq_page_attn(C.byref(c), A, A, None, A, 4, A, 1, 9, 0.125, A, 1 << 40, None) == ARG


@pytest.mark.parametrize("args", [(None, A, A, 1, None, 0), (A, None, A, 1, None, 0), (A, A, None, 1, None, 0), (A, A, A, -1, None, 0),
                                  (A, A, A, 1, None, -1), (A + 8, A, A, 1, None, 0), (A, A + 2, A, 1, None, 0), (A, A, A + 4, 1, None, 0),
                                  (A, A, A, 1, A + 2, 1), (A, A, A, 1, A, 4097)])
def test_append_refusals(kq, args):
    c = _cache(kq)
    assert kq.lib().kvq_page_append(C.byref(c), *args, None) == ARG
    assert kq.lib().kvq_page_append(None, A, A, A, 1, None, 0, None) == ARG
    assert kq.lib().kvq_page_append(C.byref(c), None, None, None, 0, None, 0, None) == 0       # nothing to do


ATTN = dict(Q=A, O=A, lse=None, tables=A, width=4, lens=A, batch=2, q_heads=9, scale=0.125, workspace=A, bytes=1 << 40)


@pytest.mark.parametrize("change", [
    dict(Q=None), dict(O=None), dict(tables=None), dict(lens=None), dict(workspace=None), dict(Q=A + 2), dict(O=A + 8), dict(lse=A + 1),
    dict(tables=A + 2), dict(lens=A + 1), dict(workspace=A + 8), dict(width=0), dict(batch=-1), dict(batch=4097), dict(q_heads=0), dict(q_heads=10),
    dict(q_heads=1), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_attention_refusals(kq, change):
    c = _cache(kq)
    assert kq.lib().kvq_page_attn(C.byref(c), *dict(ATTN, **change).values(), None) == ARG


def test_attention_refuses_other_widths_and_empty_batches_are_fine(kq):
    for d in (32, 72, 96, 256):
        c = _cache(kq, head_dim=d, slot_stride=3 * d, head_stride=d, page_stride=48 * d)
        assert kq.lib().kvq_page_attn(C.byref(c), *ATTN.values(), None) == ARG
    c = _cache(kq)
    assert kq.lib().kvq_page_attn(C.byref(c), *dict(ATTN, batch=0, tables=None, lens=None).values(), None) == 0
    n = C.c_uint64()
    for args in ((-1, 9, 3, 64), (1, 10, 3, 64), (1, 9, 3, 96), (1, 9, 0, 64)):
        assert kq.lib().kvq_page_attn_workspace_bytes(*args, C.byref(n)) == ARG
    assert kq.lib().kvq_page_attn_workspace_bytes(1, 9, 3, 64, None) == ARG


SELECT = dict(logits=A, dtype=2, scores=A, finished=None, batch=2, beams=4, vocab=100, n_out=4, end=-1, parents=A, tokens=A, scores_out=A,
              finished_out=None)


@pytest.mark.parametrize("change", [
    dict(batch=-1), dict(batch=(1 << 24) + 1), dict(beams=0), dict(beams=33), dict(n_out=0), dict(n_out=33), dict(vocab=0), dict(vocab=(1 << 30) + 1),
    dict(end=-2), dict(end=100), dict(dtype=3), dict(dtype=-1), dict(logits=None), dict(scores=None), dict(parents=None), dict(tokens=None),
    dict(scores_out=None), dict(finished=A), dict(logits=A + 2), dict(logits=A + 1, dtype=0), dict(scores=A + 2), dict(parents=A + 1),
    dict(tokens=A + 2), dict(scores_out=A + 3)])
def test_selection_refusals(kq, change):
    assert kq.lib().kvq_beam_select(*dict(SELECT, **change).values(), None) == ARG
    assert kq.lib().kvq_beam_select(*dict(SELECT, batch=0, logits=None).values(), None) == 0


@pytest.mark.parametrize("change", [
    dict(n_out=3), dict(n_out=5), dict(scores_out=A + 4), dict(scores=A + 28), dict(scores_out=A + 4096, finished=A, finished_out=A + 7, end=0),
    dict(scores_out=A + 4096, finished=A, finished_out=A, end=0, n_out=1)])
def test_selection_refuses_results_over_its_inputs(kq, change):
    """In place is fine where every request has as many beams as before (on the GPU: test_selection_in_place)."""
    assert kq.lib().kvq_beam_select(*dict(SELECT, **change).values(), None) == ARG


def test_limits_of_the_header_and_of_the_binding_agree(kq):
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "kvq.h")).read()
    for name in ("KVQ_FP16", "KVQ_BF16", "KVQ_FP32", "KVQ_MAX_PAGE_ROWS", "KVQ_MAX_PAGES", "KVQ_MAX_BEAMS", "KVQ_PAGE_FULL", "KVQ_PAGE_LONG",
                 "KVQ_PAGE_SLOTS", "KVQ_PAGE_BAD"):
        assert int(re.search(r"#define\s+%s\s+(\d+)" % name, text).group(1)) == getattr(kq, name)
    assert C.sizeof(kq.PageCache) == 64


class FakeTensor:
    """What the binding looks at of a tensor."""

    def __init__(self, dtype, count, device=0, contiguous=True):
        self.dtype, self.count, self.device, self.contiguous = dtype, count, device, contiguous

    def get_device(self):
        return self.device

    def numel(self):
        return self.count

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return A


def test_the_binding_refuses_tensors_of_another_device_type_or_size(kq):
    import torch
    assert kq._dev(FakeTensor(torch.int32, 5), torch.int32, 5, 0, "x") == A and kq._dev(None, torch.int32, 5, 0, "x") is None
    for t in (FakeTensor(torch.int32, 5, device=1), FakeTensor(torch.int32, 5, device=-1), FakeTensor(torch.int64, 5), FakeTensor(torch.int32, 4),
              FakeTensor(torch.int32, 5, contiguous=False)):
        with pytest.raises(ValueError):
            kq._dev(t, torch.int32, 5, 0, "x")
    with pytest.raises(ValueError):
        kq.kvq_page_cache(torch.zeros(2, 16, 1, 64, dtype=torch.float16), torch.zeros(2, 16, 1, 64, dtype=torch.float16))     # not on a GPU
    with pytest.raises(ValueError):
        kq.kvq_page_cache(torch.zeros(2, 16, 1, 64), torch.zeros(2, 16, 1, 64))


def test_reference_step_by_hand():
    tables = np.array([[5, 2, -1], [5, 7, -1], [1, -1, -1]])
    # rows 0 and 1 share page 5, both go on from row 0 (6 of 8 slots used): row 1 gets a copy of page 2
    out = pr.step(tables, [6, 8, 3], [0, 0, -1], [1, 3, 2], None, 9, 4, 8)
    assert out["rows"] == [[5, 2], [5, 0, 1], [3]]
    assert out["copies"] == [[-1, -1, 0], [2, 0, 2], [-1, -1, 0]]
    assert out["slots"] == [10, 2, 3, 4, 12, 13, -1, -1] and out["positions"] == [6, 6, 7, 8, 0, 1, -1, -1]
    assert out["lens"] == [7, 9, 2] and out["cu_new"] == [0, 1, 4, 6]
    assert pr.step(tables, [6, 8, 3], [0, 0, -1], [1, 3, 2], None, 9, 4, 5) is None
    assert pr.step(tables, [6, 8, 3], [0, 0, 3], [1, 3, 2], None, 9, 4, 8) is None


def test_reference_attention_and_selection_by_hand():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((2, 8)), np.zeros((5, 8)), rng.standard_normal((5, 8))
    o, lse, err, lse_err = pr.attend(q, k, v, 0.3, 11)
    assert np.allclose(o, v.mean(0)) and np.allclose(lse, np.log(5)) and np.all(err < 2e-3) and np.all(lse_err < 1e-4)
    z = np.log(np.array([[0.5, 0.25, 0.25], [0.6, 0.3, 0.1]]))
    got = pr.select(z, [-1.0, -1.0], [0, 0], 4, 2)
    assert [c[1:] for c in got] == [(1, 0, 0), (0, 0, 0), (1, 1, 0), (0, 1, 0)]
    assert np.allclose([c[0] for c in got], [-1 + np.log(x) for x in (0.6, 0.5, 0.3, 0.25)])
    assert [c[1:] for c in pr.select(z, [-9.0, -0.5], [0, 1], 2, 2)] == [(1, 2, 1), (0, 0, 0)]
