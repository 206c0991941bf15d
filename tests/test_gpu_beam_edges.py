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


# ------------------------------------------------------ what is summed again ------

def peaked(rng, m, groups):
    """Pairs of rows of a logit near m and one or two more 18 to 24 below it, whose normalizers are 2^-34 to 2^-28 apart."""
    rows = []
    while len(rows) < 2 * groups:
        first = m + rng.uniform(-1, 1, 2).astype(np.float32).astype(np.float64)
        low = rng.uniform(18, 24, 2)
        x = np.full((2, 3), -np.inf)
        x[:, 0] = np.float32(first)
        x[:, 1] = np.float32(x[:, 0] - low[0] - rng.choice([0, 0, 1]) * rng.uniform(-1, 1, 2) * 2.0 ** -rng.integers(0, 8))
        if rng.random() < 0.5:
            x[:, 2] = np.float32(x[:, 0] - low[1])
        norms = np.log1p(np.exp(x[:, 1:] - x[:, :1]).sum(1))
        if 2.0 ** -34 <= abs(norms[0] - norms[1]) <= 2.0 ** -28:
            rows += list(x)
    return np.array(rows)


@pytest.mark.parametrize("m", [0, 20, -60, 1000, -1000, 5000, 4e5])
@pytest.mark.parametrize("k", [1, 2])
def test_normalizers_that_all_but_agree(m, k):
    import torch
    rng = np.random.default_rng(abs(int(m)) + k)
    x = torch.full((600, 1024), -float("inf"), device="cuda")
    x[:, torch.tensor([17, 400, 1000], device="cuda")] = torch.tensor(peaked(rng, m, 300), dtype=torch.float32, device="cuda")
    check_select(x, np.zeros((300, 2)), k, again=False)


@pytest.mark.parametrize("vocab", [30001, 1 << 21])
@pytest.mark.parametrize("gap", [2.0 ** -34, -2.0 ** -34, 2.0 ** -31, -2.0 ** -31, 2.0 ** -28, -2.0 ** -28])
def test_long_sums_that_all_but_agree(vocab, gap):
    """Rows of one repeated logit each, where roundings add up; the second has two logits that bring it within `gap` of the first."""
    import torch
    n = vocab - 3
    low = 20 - np.log(n)                                    # the repeated ones together weigh what the largest does
    a = np.array([20.0] + [np.float32(low + 0.3)])
    b = np.array([20.0] + [np.float32(low + 0.171)])
    total = lambda x, extra=(): 1 + n * np.exp(x[1] - 20) + sum(np.exp(z - 20) for z in extra)
    want = total(a) * np.exp(gap)                           # the second's sum
    z1 = np.float64(np.float32(20 + np.log(want - total(b)) - 1e-4))
    z2 = np.float64(np.float32(20 + np.log(want - total(b, [z1]))))
    assert abs(np.log(total(b, [z1, z2]) / total(a)) / gap - 1) < 0.2
    x = torch.empty((2, vocab), device="cuda")
    x[0], x[1] = float(a[1]), float(b[1])
    x[0, 77], x[0, -2:] = 20, -float("inf")
    x[1, 9], x[1, -2], x[1, 5] = 20, z1, z2
    for k in (1, 2):
        parent, _, _ = check_select(x, np.zeros((1, 2)), k, again=False)
        assert parent[0, 0] == (0 if gap > 0 else 1)


# ------------------------------------------------- past the range of binary32 ------

LOWEST = float(np.finfo(np.float32).min)


def run(x, scores, k, done=None, end=0):
    import torch
    from paper_2608_28911_gb300 import semkv
    sc = torch.tensor(np.asarray(scores, np.float32), device="cuda")
    out = [torch.full((sc.shape[0], k), 77, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
    d = None if done is None else torch.tensor(done, dtype=torch.uint8, device="cuda")
    semkv.semkv_beam_select(x, sc, *out, semkv.beam_select_workspace(x, sc, k), done=d, end_token=end)
    return [t.cpu().numpy() for t in out]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("at", [1, 50, 700, 4000, 8999])
@pytest.mark.parametrize("beams", [1, 128])
def test_scores_below_the_lowest_number(dtype, at, beams):
    """A finite logit is a candidate however far it lies below the largest, in whichever thread's vectors."""
    import torch
    dt = getattr(torch, dtype)
    x = torch.full((beams, 9000), -float("inf"), dtype=dt, device="cuda")
    b = beams - 1
    x[b, 0], x[b, at] = 3e38, -3e38
    s = np.full((1, beams), -np.inf)
    s[0, b] = -1
    parent, token, score = run(x, s, 3)
    assert parent.tolist() == [[b, b, -1]] and token.tolist() == [[0, at, -1]]
    assert score[0].tolist() == [-1.0, LOWEST, -np.inf]


def test_scores_below_the_lowest_number_of_two_beams():
    """Whatever they would be: the lower row first, then the larger logit, then the lower token."""
    import torch
    x = torch.full((2, 5000), -float("inf"), device="cuda")
    x[0, 9], x[0, 4000], x[0, 4001], x[0, 20] = 3.2e38, -3.1e38, -3e38, -3.1e38
    x[1, 8], x[1, 7], x[1, 3000] = 1.0, -3.1e38, -3.4e38
    parent, token, score = run(x, [[-2, -3.1e38]], 8)
    want = [(0, 9), (1, 8), (0, 4001), (0, 20), (0, 4000), (1, 7), (1, 3000), (-1, -1)]
    assert list(zip(parent[0].tolist(), token[0].tolist())) == want
    assert score[0].tolist() == [-2.0, np.float32(-3.1e38)] + [LOWEST] * 5 + [-np.inf]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("vocab", [700, 40001])
def test_a_beam_at_the_lowest_score(dtype, vocab):
    """Tokens masked by the type's lowest number.  What lies below binary32's range comes behind all that does not."""
    import torch
    dt = getattr(torch, dtype)
    x = torch.full((3, vocab), torch.finfo(dt).min, dtype=dt, device="cuda")
    x[0, 77], x[2, 5], x[2, 600] = 3, 1, 2
    for k in (2, 20, 128):
        parent, token, score = run(x, [[LOWEST, -np.inf, -np.inf]], k)
        assert (parent == 0).all() and (score == LOWEST).all()
        assert token[0].tolist() == [77] + [t for t in range(128) if t != 77][:k - 1]
        parent, token, score = run(x, [[LOWEST, -np.inf, -2.0]], k)
        # the masked ones of the third row are near that type's lowest number; in binary32 a little below the first row's best
        want = [(2, 600), (2, 5)] + ([(0, 77)] if dtype == "float32" else []) + [(2, t) for t in range(140) if t != 5]
        assert list(zip(parent[0].tolist(), token[0].tolist())) == want[:k]
    parent, token, score = run(x, [[LOWEST, -2.0, LOWEST]], 4, done=[0, 0, 1], end=9)
    assert (parent[0] == 1).all() and token[0].tolist() == [0, 1, 2, 3]
