"""The selection of beams where single numbers go wrong: scores of great size (GPU)."""
import math

import numpy as np
import pytest

import pages_reference as pr
from test_gpu_beams import _check, _dtypes, _logits, _run, _scores

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


FAR = [-1e9, -1e17, -1e25, -1e30, float(np.finfo(np.float32).min)]


def _check_far(logits, scores, n, got):
    """Beams of scores so large that fp64 cannot tell their candidates apart: as many as there are, each once, best first, every score
    to the rounding of fp64 at its size; none that is left out is better than the last by more."""
    parents, tokens, out, over = got
    z = logits.float().cpu().numpy().astype(np.float64)
    B, W, V = z.shape
    for b in range(B):
        there = np.isfinite(z[b])
        top = np.where(there, z[b], -np.inf).max(1, keepdims=True)
        logp = z[b] - top - np.log(np.exp(z[b] - top).sum(1, keepdims=True))
        score = np.asarray(scores[b], np.float64)[:, None] + logp
        slack = 2.0 ** -51 * np.abs(score) + 2.0 ** -17
        k = min(n, int(there.sum()))
        assert np.all(parents[b, :k] >= b * W) and np.all(parents[b, k:] == -1), (b, parents[b])
        w, t = parents[b, :k] - b * W, tokens[b, :k]
        assert len(set(zip(w.tolist(), t.tolist()))) == k
        best = np.sort(score[there])[::-1][:k]
        assert np.all(np.abs(score[w, t] - best) <= slack[w, t]), b
        assert np.all(np.abs(out[b, :k] - best) <= slack[w, t] + 2.0 ** -24 * np.abs(best))


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("score", FAR)
@pytest.mark.parametrize("B,W,V,n", [(1, 1, 1000, 4), (2, 1, 30011, 32), (1, 4, 7, 20), (3, 5, 5001, 5), (200, 3, 600, 7)])
def test_beams_of_very_low_scores_have_all_their_candidates(kq, B, W, V, n, score, kind):
    z = _logits(V + n, B, W, V, _dtypes()[kind])
    s = np.full((B, W), score, np.float32)
    _check_far(z, s, n, _run(kq, z, s, None, n, -1))


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("score", FAR)
def test_a_masked_first_beam_beside_beams_of_very_low_scores(kq, score, kind):
    """One beam takes part and a mask leaves it two tokens: the rest come from the others."""
    z = _logits(9, 4, 4, 2003, _dtypes()[kind])
    z[:, 0, 2:] = -math.inf
    s = np.full((4, 4), score, np.float32)
    s[:, 0] = 0.0
    got = _run(kq, z, s, None, 4, -1)
    assert np.all(got[0][:, :2] == np.arange(4)[:, None] * 4) and np.all(got[0][:, 2:] % 4 > 0)
    _check_far(z, s, 4, got)


@pytest.mark.parametrize("score", FAR[3:])
def test_scores_that_fp64_does_not_tell_apart_are_ties(kq, score):
    """Where a score swallows every logit the lowest beams and tokens win."""
    for kind, V in ((0, 40), (1, 3001), (2, 50000)):
        z = _logits(V, 2, 3, V, _dtypes()[kind])
        for n in (1, 5, 32):
            parents, tokens, out, _ = _run(kq, z, np.full((2, 3), score, np.float32), None, n, -1)
            assert parents.tolist() == [[3 * b] * n for b in range(2)] and tokens.tolist() == [list(range(n))] * 2
            assert np.all(out == np.float32(score))
