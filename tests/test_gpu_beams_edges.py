"""The selection of beams where single numbers go wrong: scores of great size, sums of very many entries, rows that rise from end
to end (GPU)."""
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


def _sum_error(kq, z):
    """How far each beam's logarithm of its sum of exponentials is off, from the scores of its candidates (in fp64 but for their last rounding)."""
    import torch
    B, W, V = z.shape
    parents, tokens, out, _ = _run(kq, z, np.zeros((B, W), np.float32), None, W, -1)
    worst = 0.0
    for b in {0, B // 2, B - 1}:
        x = z[b].double()
        want = (x - torch.logsumexp(x, 1, keepdim=True)).cpu().numpy()
        for p, t, s in zip(parents[b], tokens[b], out[b].astype(np.float64)):
            exact = want[p - b * W, t]
            worst = max(worst, abs(s - exact) - 2.0 ** -24 * abs(exact))
    return worst


@pytest.mark.parametrize("rise", [0.5, 4.0, 30.0, 400.0])
@pytest.mark.parametrize("B,W,V", [(1, 32, 1 << 20), (300, 17, 40000), (1, 4, 3000000)])
def test_sums_of_rows_that_rise_from_end_to_end(kq, B, W, V, rise):
    """A warp's reference moves up chunk by chunk.  Errors per entry: its distance d to the reference in log2 units three times rounded, 2.25 |d| 2^-24 ln 2,
    where the mean of |d| is at most log2 V + 6 (entropy, and a reference that lies up to 4 nats low); the exponential's own 2^-22, once more for
    each of the five or fewer times that the reference moves by 4 and still matters, and for the lanes' join; eight fp32 additions, 8 x 2^-24.  For
    V = 2^22 that is (2.25 x 0.694 x 28 + 4 x 7 + 8) 2^-24 = 80 x 2^-24."""
    import torch
    row = torch.linspace(0, rise, V, device="cuda")
    z = torch.stack([row + 0.01 * w for w in range(W)])[None].expand(B, W, V).contiguous()
    assert _sum_error(kq, z) <= 80 * 2.0 ** -24


@pytest.mark.parametrize("gap", [9.3, 11.0, 11.7, 12.4, 13.9, 15.3])
def test_sums_of_flat_rows_under_one_peak(kq, gap):
    """All entries but one have the same distance from the reference and so the same error: the bound above without moves."""
    import torch
    z = torch.full((1, 32, 1 << 20), 0.0, device="cuda") + torch.linspace(-0.3, 0.3, 32, device="cuda")[None, :, None]
    z[:, :, 777] += gap
    assert _sum_error(kq, z) <= 60 * 2.0 ** -24


def test_scores_below_the_range_of_fp32(kq):
    """A candidate counts while its score is finite in fp64; it is returned as -inf, with its beam and token, if fp32 does not hold it."""
    import torch
    low = float(np.finfo(np.float32).min)
    z = torch.tensor([[[low, 1.0, -math.inf, 0.5, low]]], device="cuda")
    parents, tokens, out, over = _run(kq, z, np.full((1, 1), low, np.float32), None, 6, 3)
    assert tokens[0].tolist() == [1, 3, 0, 4, -1, -1] and parents[0].tolist() == [0, 0, 0, 0, -1, -1] and over[0].tolist() == [0, 1, 0, 0, 1, 1]
    assert out[0].tolist() == [low, low] + [-math.inf] * 4
