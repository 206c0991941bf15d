"""Selections where little decides: scores that lie within a rounding of one another, whatever their rows' logits and
their own sizes.  Every index is that of the definition."""
import numpy as np
import pytest

from test_gpu_search import check_select

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------- what is looked at ------

def ties_beside_one(dt, far, beams, ties, where):
    """Groups of two beams that are read, at where[0] and where[1]: one has a single candidate, the other `ties` of the same
    logit, in threads of their own and more of them than a threshold lets through beside k.  Either's logit is
    `far`, the other's 0, and the scores are a little apart, either way."""
    import torch
    logit = float(torch.tensor(far, dtype=dt))
    rows, scores = [], []
    for m in (logit, -logit):
        for gap in (1, -1, 0.3, -0.3, 0.1, -0.1, 0.03, -0.03):
            for one, many in ((m, 0.0), (0.0, m)):
                x = torch.full((beams, 1024), -float("inf"), dtype=dt)
                s = np.full(beams, -np.inf, np.float32)
                x[where[0], 5] = one
                x[where[1], torch.arange(ties) * 8] = many
                s[where[0]] = -5
                s[where[1]] = -5 + np.log(ties) + gap * abs(m) * 2.0 ** -24
                assert abs(float(s[where[1]]) - np.log(ties) + 5) > 2.0 ** -34
                rows.append(x), scores.append(s)
    return torch.cat(rows).cuda(), np.stack(scores)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("k,ties", [(1, 20), (17, 40)])
@pytest.mark.parametrize("beams,where", [(2, (0, 1)), (2, (1, 0)), (128, (3, 100))])
def test_rows_of_far_logits_beside_others(dtype, k, ties, beams, where):
    import torch
    for far in (100, 300, 1000, 5001, 10007, 36640, 65000, 100003, 300007, 900007, 2 ** 20 - 1, 2 ** 20):
        if dtype != "float16" or far < 65504:
            check_select(*ties_beside_one(getattr(torch, dtype), far, beams, ties, where), k, again=False)


def test_two_far_logits_by_hand():
    import torch
    ninf = -float("inf")
    for dt, far, score, first in ((torch.float32, 900007, -1.9969914, 1), (torch.float16, 36640, -2.0049002, 0)):
        x = torch.full((2, 1024), ninf, dtype=dt, device="cuda")
        x[0, 0] = far
        x[1, torch.arange(20) * 8] = 0
        parent, token, _ = check_select(x, np.array([[-5, score]]), 1)
        assert (parent[0, 0], token[0, 0]) == (first, 0)


@pytest.mark.parametrize("k,beams", [(3, 2), (18, 2), (18, 128)])
def test_scores_above_zero_that_logits_bring_back(k, beams):
    """Twenty candidates (forty) of a beam at a large score come out near 0, as the one of a beam that stands there does."""
    import torch
    ties, rows, scores = 20 if k == 3 else 40, [], []
    for big in (1e3, 1e5, 1e6, 3e7):
        # beside the first two the ties weigh nothing: the row's norm is ln(1 + exp(-1/2))
        base = np.float64(np.float32(big)) - np.log1p(np.exp(-0.5))
        for logit in np.float32(-big) + np.spacing(np.float32(big)) * np.arange(-2, 4):
            tie = base + np.float64(logit)
            for gap in (0.3, -0.3, 0.05, -0.05, 0.01, -0.01):
                x = torch.full((beams, 1024), -float("inf"))
                x[0, 1], x[0, 1021] = 0, -0.5
                x[0, torch.arange(ties) * 8 + 32] = float(logit)
                x[1, 7] = 3
                s = np.full(beams, -np.inf, np.float32)
                s[0], s[1] = big, tie + gap * np.spacing(np.float32(big))
                assert abs(tie - np.float64(s[1])) > 2.0 ** -20 * abs(tie)
                rows.append(x), scores.append(s)
    check_select(torch.cat(rows).cuda(), np.stack(scores), k, again=False)
