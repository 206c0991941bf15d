"""Selections where little decides: scores that lie within a rounding of one another, whatever their rows' logits and
their own sizes, and calls that are cut into long or very many pieces.  Every index is that of the definition."""
import numpy as np
import pytest

from test_gpu_search import check_select, score_bound

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


# ------------------------------------------------------ long and many pieces ------

def cut(rows, vocab, dtype, aligned):
    """Units of a row, units of a CTA's share, pieces of a row: the rule that rows are cut by."""
    per = 4 if dtype == "float32" else 8
    unit = 256 * per
    units = -(-(vocab + (0 if aligned else per - 1)) // unit)
    share = -(-rows * units // 608)
    if units >= 4:
        share = -(-share // 4) * 4
    if share < units < 8:
        share = units
    share = min(share, 128)
    return units, share, units // share if units % share == 0 else (units + share - 2) // share + 1


def is_cut_so(groups, beams, vocab, dtype, aligned, pieces):
    """By the rule, and by the size of the library's workspace: 3088 bytes for each piece, however rows lie."""
    import torch
    from paper_2608_28911_gb300 import semkv
    rows = groups * beams
    size = semkv.semkv_beam_select_workspace_bytes(groups, beams, vocab, getattr(torch, dtype), 128)
    most = max(cut(rows, vocab, dtype, a)[2] for a in (True, False))
    return cut(rows, vocab, dtype, aligned) == pieces and size == rows * most * (16 + 256 * 12)


def best_of_rows(x):
    """Each row's 128 best tokens with their log probabilities in 64 bits, by a stable sort on the GPU."""
    import torch
    tokens, values = [], []
    for row in x:
        best, at = row.float().sort(descending=True, stable=True)
        norm = (row.double() - best[0]).exp_().sum().log()
        tokens.append(at[:128]), values.append((best[:128].double() - best[0]) - norm)
    return torch.stack(tokens).cpu(), torch.stack(values).cpu()


def check_by(best, x, scores, k, done=None, end=0):
    """A selection against best = best_of_rows(x)."""
    import torch
    from paper_2608_28911_gb300 import semkv
    groups, beams = scores.shape
    sc = torch.tensor(np.asarray(scores, np.float32), device="cuda")
    d = None if done is None else torch.tensor(np.asarray(done, np.uint8), device="cuda")
    ws = semkv.beam_select_workspace(x, sc, k)
    ws.fill_(255)
    out = [torch.full((groups, k), 77, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
    semkv.semkv_beam_select(x, sc, *out, ws, done=d, end_token=end)
    parent, token, score = [t.cpu() for t in out]
    sc = sc.double().cpu().view(-1)
    for g in range(groups):
        rows, tokens, values = [], [], []
        for r in range(g * beams, (g + 1) * beams):
            if sc[r] == -np.inf:
                continue
            over = done is not None and done[r]
            values.append(sc[r:r + 1] if over else best[1][r] + sc[r])
            tokens.append(torch.tensor([end]) if over else best[0][r])
            rows.append(torch.full((len(tokens[-1]),), r))
        rows, tokens, values = torch.cat(rows), torch.cat(tokens), torch.cat(values)
        order = values.sort(descending=True, stable=True)[1][:k]
        n = len(order)
        wrong = (parent[g, :n] != rows[order]) | (token[g, :n] != tokens[order])
        assert not wrong.any(), (g, k, wrong.nonzero()[:3].tolist())
        assert ((score[g, :n].double() - values[order]).abs() <= torch.tensor(score_bound(x.shape[1], values[order].numpy()))).all()
        assert (parent[g, n:] == -1).all()


def fill_rows(x, kinds, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    vocab = x.shape[1]
    ramp = torch.linspace(-9, 9, vocab, device="cuda")
    for r in range(len(x)):
        kind = kinds[r % len(kinds)]
        x[r] = {"random": lambda: torch.randn(vocab, generator=gen, device="cuda") * 3, "rising": lambda: ramp, "falling": lambda: -ramp,
                "equal": lambda: torch.full_like(ramp, 1.25), "steps": lambda: (4 * ramp).round() / 4}[kind]().to(x.dtype)


KINDS = [["random"], ["rising"], ["falling"], ["equal"], ["steps"], ["random", "rising", "equal", "falling", "steps"]]


@pytest.mark.parametrize("dtype,groups,beams,vocab,pad,pieces", [
    ("bfloat16", 64, 16, 131072, 0, (64, 108, 2)), ("bfloat16", 64, 16, 131071, 0, (65, 112, 2)), ("float16", 5, 16, (1 << 21) - 3, 1, (1025, 128, 9)),
    ("float32", 3, 16, (1 << 21) + 8, 3, (2049, 128, 17)), ("bfloat16", 65, 20, 24576, 0, (12, 28, 2)), ("float32", 65, 20, 12291, 2, (13, 28, 2))])
def test_shares_of_many_tiles(dtype, groups, beams, vocab, pad, pieces):
    """Up to 32 tiles of four units each, shares that end anywhere in a row and hold several."""
    import torch
    assert is_cut_so(groups, beams, vocab, dtype, (vocab + pad) * (4 if dtype == "float32" else 2) % 16 == 0, pieces)
    x = torch.empty((groups * beams, vocab + pad), dtype=getattr(torch, dtype), device="cuda")[:, :vocab]
    rng = np.random.default_rng(vocab)
    for i, kinds in enumerate(KINDS):
        fill_rows(x, kinds, i)
        best = best_of_rows(x)
        for k in (1, 32, 128):
            check_by(best, x, rng.uniform(-3, -2, (groups, beams)), k)


def test_more_pieces_than_a_table_holds():
    """The best beams among the last, rows of every kind, done ones, and beams of which all or few have a chance."""
    import torch
    beams, vocab = 128, 1100000
    splits = 10
    assert is_cut_so(1, beams, vocab, "float32", True, (1075, 128, splits)) and beams * splits > 1024
    last = 1024 // splits + 2                     # all pieces from this beam on lie past the first table
    x = torch.empty((beams, vocab), device="cuda")
    rng = np.random.default_rng(3)
    done = np.zeros(beams, int)
    done[[5, 60, last + 3]] = 1
    for i, kinds in enumerate(KINDS):
        fill_rows(x, kinds, i)
        best = best_of_rows(x)
        for k in (1, 17, 128):
            near = rng.uniform(-3, -2, (1, beams))
            check_by(best, x, near, k)
            check_by(best, x, near - 20.0 * (np.arange(beams) < last), k)
            check_by(best, x, np.where(np.arange(beams) == last + 5, near, -np.inf), k, done, 99)
            check_by(best, x, near - 20.0 * (np.arange(beams) != last + 1), k, done, 99)


# ------------------------------------------------------------ behind the ends ------

class Fence:
    """Tensors with known bytes before and behind them."""

    def __init__(self):
        self.held = []

    def bytes(self, n):
        import torch
        store = torch.full((512 + n + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
        self.held.append((store, n))
        return store[512:512 + n]

    def like(self, shape, dtype):
        import torch
        return self.bytes(int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()).view(dtype).view(shape)

    def whole(self):
        return all(bool((s[:512] == 0xA5).all()) and bool((s[512 + n:] == 0xA5).all()) for s, n in self.held)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("groups,beams,vocab,k", [(1, 1, 1, 1), (1, 4, 32768, 8), (5, 5, 50003, 10), (3, 7, 2049, 128), (1, 128, 9000, 128),
                                                  (700, 2, 5000, 5), (1, 64, 100003, 33), (64, 16, 4099, 16)])
def test_selections_stay_within_their_tensors(dtype, groups, beams, vocab, k):
    import torch
    from paper_2608_28911_gb300 import semkv
    dt = getattr(torch, dtype)
    rng = np.random.default_rng(vocab)
    gen = torch.Generator(device="cuda").manual_seed(k)
    for lead, pad in ((0, -vocab % 8), (0, 1 - vocab % 2), (3, 2 - vocab % 2)):
        store = torch.randn(lead + groups * beams * (vocab + pad), generator=gen, device="cuda").to(dt)
        x = store[lead:].view(groups * beams, vocab + pad)[:, :vocab]
        scores = torch.tensor(rng.uniform(-3, -2, (groups, beams)).astype(np.float32), device="cuda")
        plain = [torch.empty((groups, k), dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
        semkv.semkv_beam_select(x, scores, *plain, semkv.beam_select_workspace(x, scores, k))
        f = Fence()
        out = [f.like((groups, k), t) for t in (torch.int32, torch.int32, torch.float32)]
        ws = f.bytes(semkv.semkv_beam_select_workspace_bytes(groups, beams, vocab, dt, k))
        semkv.semkv_beam_select(x, scores, *out, ws)
        assert all(torch.equal(a, b) for a, b in zip(out, plain))
        assert f.whole()


@pytest.mark.parametrize("wide", [0, 300, 9000])
def test_reorders_stay_within_their_tensors(wide):
    import torch
    from search_plain import reorder
    from test_gpu_kv4 import fill, make, t32
    from paper_2608_28911_gb300 import semkv
    rng = np.random.default_rng(4)
    lens = [int(v) for v in rng.integers(0, 200, 60)]
    c = make(lens, 1, 64, 16, spare=0, seed=2, more_pages=wide)
    plain = fill(c)
    for n in (60, 17, 1):
        f = Fence()
        ws = f.bytes(c.pages_workspace(n, 0).numel())
        seqs, parent = rng.permutation(60)[:n], rng.integers(-1, n, n)
        semkv.semkv_kv4_reorder(c, t32(seqs), t32(parent), ws)
        reorder(plain, seqs, parent)
        plain.same_state(c)
        assert f.whole()
