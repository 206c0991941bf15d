"""A search step over the paged 4-bit cache on the GPU against its definitions on the host (search_plain.py):
rotated rows and page states equal in every byte, selections equal in every index, scores within bounds derived
from their roundings, and the calls together as a search makes them."""
import numpy as np
import pytest

from kv4_plain import Plain
from search_plain import reorder, select, table_of, turn
from test_gpu_kv4 import SPECIAL, cu_of, fill, make, rows_like, t32

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------- rotated rows ------

def bare(pages, D):
    """Code bytes without the sign of zero codes (it is the value's own)."""
    codes = pages[..., :16 * D].copy()
    codes &= np.where(codes & 0x0F == 0x08, 0xF0, 0xFF).astype(np.uint8)
    codes &= np.where(codes & 0xF0 == 0x80, 0x0F, 0xFF).astype(np.uint8)
    return codes


def same_pages(c, plain, layer):
    D, got = c.s.head_dim, c.pages.cpu().numpy()
    assert np.array_equal(got[..., 16 * D:], plain.pages[..., 16 * D:])
    same = bare(got, D) == bare(plain.pages, D)
    assert same.all(), np.argwhere(~same)[:5]
    others = [i for i in range(len(got)) if i != layer]
    assert np.array_equal(got[others], plain.pages[others])


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("D,P,H,group,rot", [(128, 64, 2, 4, 128), (128, 16, 3, 1, 64), (64, 32, 1, 7, 64), (64, 128, 5, 2, 16),
                                             (128, 32, 1, 16, 48), (64, 16, 2, 3, 32)])
@pytest.mark.parametrize("own_positions", [False, True])
def test_rows_are_turned_and_stored_as_defined(dtype, pairs, D, P, H, group, rot, own_positions):
    import torch
    from paper_2608_28911_gb300 import semkv
    dt = getattr(torch, dtype)
    lens, counts = [0, 1, 40, 129, 16, 77], [0, 1, 7, 129, 16, 30]
    c = make(lens, H, D, P, layers=2, seed=D + P)
    plain = Plain(c)
    rng = np.random.default_rng(3)
    total, Hq = sum(counts) + 5, H * group       # five rows that belong to nobody
    wide = rows_like(rng, (total, Hq + 2 * H + 1, D), dt)     # Q, K and V in one row, and something behind
    flat = wide.view(-1)
    flat[torch.tensor(rng.integers(0, flat.numel(), 60), device="cuda")] = torch.tensor(SPECIAL * 6, dtype=dt, device="cuda")
    q, k, v = wide[:, :Hq], wide[:, Hq:Hq + H], wide[:, Hq + H:Hq + 2 * H]
    k[3, :, 16:32] = 0
    seqs = [3, 1, 0, 5, 2, 4]
    counts = [counts[s] for s in seqs]
    start = [lens[s] - n for s, n in zip(seqs, counts)]
    start[1] = -1                                 # left out
    b = semkv.KV4Batch(6, cu=cu_of(counts), seqs=t32(seqs), start=t32(start), total=total, max_count=200)
    table = table_of(300, rot)
    place = np.concatenate([p + np.arange(n) for p, n in zip(start, counts)] + [np.zeros(5, int)])
    position = rng.integers(0, 300, total) if own_positions else place
    if own_positions:
        position[[2, 9, 150]] = -1, 300, 2 ** 31 - 1          # rows without an angle
    r = semkv.KV4Rotation(torch.tensor(table, device="cuda"), pairs)
    out = torch.full((total, Hq + 1, D), 7.0, dtype=dt, device="cuda")[:, :Hq]
    semkv.semkv_kv4_write_rotated(c, b, 1, r, k, v, q, out, positions=t32(position) if own_positions else None)
    angles = table[np.clip(position, 0, 299)]
    qf, kf = [turn(x.float().cpu().numpy(), angles, rot, pairs) for x in (q, k)]
    vf = v.float().cpu().numpy()
    want = torch.tensor(qf).to(dt).float().numpy()
    row, there = 0, np.zeros(total, bool)
    for s, n, p in zip(seqs, counts, start):
        for j in range(n if p >= 0 else 0):
            if 0 <= position[row + j] < 300:
                plain.write(1, s, p + j, kf[row + j], vf[row + j])
                there[row + j] = True
        row += n
    want[~there] = 7
    assert np.array_equal(out.float().cpu().numpy(), want, equal_nan=True)
    same_pages(c, plain, 1)
    told = {3} if own_positions else set()         # rows without an angle, and keys and values that are no numbers
    if not (np.isfinite(kf[there]).all() and np.isfinite(vf[there]).all()):
        told.add(4)
    assert int(c.dev_error.item()) in (told or {0})
    # in place, and the keys and values alone, into the same pages
    c.pages.fill_(255)
    semkv.semkv_kv4_write_rotated(c, b, 1, r, k, v, positions=t32(position) if own_positions else None)
    same_pages(c, plain, 1)
    before = q.clone()
    semkv.semkv_kv4_write_rotated(c, b, 1, r, k.clone(), v.clone(), q, q, positions=t32(position) if own_positions else None)
    there = torch.tensor(there, device="cuda")
    assert np.array_equal(q[there].float().cpu().numpy(), want[there.cpu().numpy()], equal_nan=True)
    assert np.array_equal(q[~there].float().cpu().numpy(), before[~there].float().cpu().numpy(), equal_nan=True)


@pytest.mark.parametrize("n,H,group", [(1, 8, 4), (64, 8, 4), (300, 1, 1), (1, 1, 128)])
def test_a_turned_row_is_the_written_one(n, H, group):
    """Without an angle (cosine 1, sine 0) the call writes what semkv_kv4_write does, and a query stays."""
    import torch
    from paper_2608_28911_gb300 import semkv
    c = make([50] * n, H, 128, 32, seed=n)
    rng = np.random.default_rng(n)
    q, k, v = [rows_like(rng, (n, h, 128), torch.bfloat16) for h in (H * group, H, H)]
    b = semkv.KV4Batch(n, start=t32([49] * n))
    semkv.semkv_kv4_write(c, b, 0, k, v)
    want = c.pages.clone()
    c.pages.fill_(255)
    flat = torch.cat((torch.ones((50, 64)), torch.zeros((50, 64))), 1).cuda()
    out = torch.empty_like(q)
    semkv.semkv_kv4_write_rotated(c, b, 0, semkv.KV4Rotation(flat), k, v, q, out)
    assert torch.equal(out, q) and torch.equal(c.pages, want) and int(c.dev_error.item()) == 0


def test_rotated_rows_without_a_place_are_left_out():
    import torch
    from paper_2608_28911_gb300 import semkv
    c = make([40, 40, 40], H=1, D=64, P=16, spare=0)
    c.table[1, 1] = c.s.num_pages                # a page that is not there
    before = c.pages.clone()
    k = torch.ones((4, 1, 64), dtype=torch.float16, device="cuda")
    r = semkv.KV4Rotation(torch.ones((4000, 64), device="cuda"))
    for seqs, start in (([7, -1, 3, 1], [0, 0, 0, 20]), ([0, 1, 2, 0], [48, 17, 1000, 2 ** 31 - 1])):
        c.dev_error.zero_()
        b = semkv.KV4Batch(4, seqs=t32(seqs), start=t32(start))
        out = torch.full_like(k, 7.0)
        semkv.semkv_kv4_write_rotated(c, b, 0, r, k, k, k, out, positions=t32([0, 1, 2, 3]))
        assert torch.equal(c.pages, before) and (out == 7).all() and int(c.dev_error.item()) == 3


def test_rotated_rows_in_graphs_and_on_streams():
    """A step's reserve and append, captured and replayed on new rows, against eager calls on a stream."""
    import torch
    from paper_2608_28911_gb300 import semkv
    rng = np.random.default_rng(6)
    rot = semkv.KV4Rotation(torch.tensor(table_of(64, 64), device="cuda"))
    caches = [make([5, 31, 0], 2, 64, 32, spare=6, seed=4, more_pages=1) for _ in range(2)]
    for c in caches:
        c.pages.zero_()
    steps = [semkv.KV4Batch(3) for _ in caches]
    rows = [[rows_like(rng, (3, h, 64), torch.bfloat16) for h in (2, 2, 6)] for _ in range(4)]
    k, v, q = [x.clone() for x in rows[0]]
    outs = [torch.empty_like(q) for _ in caches]
    spaces = [c.pages_workspace(3) for c in caches]

    def step(i, k, v, q, **kw):
        semkv.semkv_kv4_reserve(caches[i], steps[i], spaces[i], **kw)
        semkv.semkv_kv4_write_rotated(caches[i], steps[i], 0, rot, k, v, q, outs[i], **kw)

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(0, k, v, q)
    stream = torch.cuda.Stream()
    for new in rows:
        for to, x in zip((k, v, q), new):
            to.copy_(x)
        g.replay()
        torch.cuda.synchronize()
        step(1, *new, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(caches[0].pages, caches[1].pages)
        assert torch.equal(caches[0].length, caches[1].length)
    assert int(caches[0].dev_error.item()) == int(caches[1].dev_error.item()) == 0
    assert caches[0].length.tolist() == [9, 35, 4]


# -------------------------------------------------------------- beam selection ------

def score_bound(vocab, want):
    """A normalizer's error as the kernel counts it, in units of 2^-24: exponents' arguments are off by half a step, 1
    for each of |x - m| + 3 ln 2 and 1.125 with what log2 e lacks, at most ln vocab on the average; the exponentials
    by 4, sums of eight and of four numbers by 5, the logarithm by 1; and half a step of the score's own rounding."""
    with np.errstate(invalid="ignore"):
        return (1.125 * np.log(vocab) + 13.5) * 2.0 ** -24 + 2.0 ** -24 * np.abs(want)


def check_select(logits, scores, k, done=None, end=0, error=0, again=True):
    """Runs a selection and compares it; logits a GPU tensor [rows][vocab]."""
    import torch
    from paper_2608_28911_gb300 import semkv
    groups, beams = scores.shape
    sc = torch.tensor(np.asarray(scores, np.float32), device="cuda")
    d = None if done is None else torch.tensor(np.asarray(done, np.uint8), device="cuda")
    ws = semkv.beam_select_workspace(logits, sc, k)
    ws.fill_(255)
    err = t32([0])
    out = [torch.full((groups, k), 77, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
    semkv.semkv_beam_select(logits, sc, *out, ws, done=d, end_token=end, dev_error=err)
    assert int(err.item()) == error
    parent, token, score = [t.cpu().numpy() for t in out]
    wp, wt, wsc = select(logits.double().cpu().numpy(), sc.double().cpu().numpy(), k, done, end)
    assert np.array_equal(parent, wp) and np.array_equal(token, wt), (np.argwhere((parent != wp) | (token != wt))[:5], score[:2], wsc[:2])
    assert np.array_equal(np.isinf(score), np.isinf(wsc))
    fin = np.isfinite(wsc)
    off = np.abs(score[fin] - wsc[fin]) - score_bound(logits.shape[1], wsc[fin])
    assert (off <= 0).all(), off.max()
    if again:
        more = [torch.empty_like(t) for t in out]
        semkv.semkv_beam_select(logits, sc, *more, ws, done=d, end_token=end)
        assert all(torch.equal(a, b) for a, b in zip(out, more))
    return parent, token, score


def logits_like(rng, rows, vocab, dtype, pad=0, width=3.0):
    import torch
    x = torch.tensor(rng.standard_normal((rows, vocab + pad)) * width, device="cuda").to(dtype)
    return x[:, :vocab]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("vocab,pad", [(1, 0), (2, 5), (7, 0), (100, 3), (1023, 0), (1025, 1), (2048, 0), (8191, 4), (8193, 7), (50003, 0)])
@pytest.mark.parametrize("groups,beams,k", [(1, 1, 1), (2, 4, 8), (3, 5, 10), (1, 17, 128)])
def test_selections(dtype, vocab, pad, groups, beams, k):
    import torch
    rng = np.random.default_rng(vocab + 31 * beams)
    x = logits_like(rng, groups * beams, vocab, getattr(torch, dtype), pad)
    check_select(x, rng.uniform(-8, -2, (groups, beams)), k)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("groups,beams,vocab,k", [(5, 128, 1000, 128), (40, 3, 4000, 1), (1, 2, 400000, 128), (130, 16, 600, 32), (2, 64, 33000, 64)])
def test_selections_with_many_of_something(dtype, groups, beams, vocab, k):
    import torch
    rng = np.random.default_rng(groups)
    x = logits_like(rng, groups * beams, vocab, getattr(torch, dtype), 3, 1.0)
    check_select(x, rng.uniform(-3, -2, (groups, beams)), k)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_rows_in_any_order_of_their_values(dtype):
    """Ascending, descending, constant rows, and rows of a few values: ties go to the lower token."""
    import torch
    dt = getattr(torch, dtype)
    vocab = 70001
    ramp = torch.linspace(-20, 20, vocab, device="cuda")
    rng = np.random.default_rng(2)
    few = torch.tensor(rng.integers(0, 3, vocab), device="cuda").float()
    steps = torch.arange(vocab, device="cuda").float() * 2.0 ** -9 - 100    # one more bit each, for long
    for rows in ([ramp], [-ramp], [torch.zeros_like(ramp)], [few], [steps], [ramp, few, -ramp, ramp * 0, steps]):
        x = torch.stack(rows).to(dt)
        for k in (1, 8, 100, 128):
            check_select(x, np.arange(len(rows))[None] * -0.2371, k)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("groups,beams,vocab,k", [(1, 8, 1100000, 128), (1, 64, 100003, 128), (2, 128, 30000, 16)])
def test_long_rows_in_any_order_of_their_values(dtype, groups, beams, vocab, k):
    """Many pieces with many tiles each, whose logits rise all along, fall, or repeat."""
    import torch
    dt = getattr(torch, dtype)
    rng = np.random.default_rng(vocab)
    x = torch.empty((groups * beams, vocab), dtype=dt, device="cuda")
    ramp = torch.linspace(-9, 9, vocab, device="cuda")
    for r in range(len(x)):
        x[r] = [ramp, -ramp, ramp.round(), torch.tensor(rng.standard_normal(vocab), device="cuda")][r % 4].to(dt)
    check_select(x, rng.uniform(-3, -2, (groups, beams)), k, again=False)
    check_select(x, np.where(np.arange(groups * beams).reshape(groups, beams) % 5 == 3, -1.0, -1e9), k, again=False)


def test_equal_rows_and_equal_scores():
    """Beams that are alike: the lower one first, and wherever a row lies its sum is the same."""
    import torch
    rng = np.random.default_rng(7)
    row = torch.tensor(rng.standard_normal(5003) * 3, device="cuda")
    for dtype in (torch.float16, torch.bfloat16, torch.float32):
        x = torch.empty((12, 5003), dtype=dtype, device="cuda")   # an odd stride: rows lie at all offsets
        x[:] = row.to(dtype)
        parent, token, _ = check_select(x, np.full((2, 6), -1.5), 40)
        assert parent[0, :6].tolist() == [0, 1, 2, 3, 4, 5] and len(set(token[0, :6])) == 1


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_scores_that_all_but_agree(dtype):
    """Two beams' best candidates closer than a binary32 sum's error: the order is the exact one."""
    import torch
    dt = getattr(torch, dtype)
    rng = np.random.default_rng(11)
    near = 0
    for _ in range(40):
        x = logits_like(rng, 2, 30011, dt)
        xd = x.double()
        best = (xd.amax(1) - torch.logsumexp(xd, 1)).cpu().numpy()
        scores = np.array([[0.0, np.float32(best[0] - best[1])]], np.float32)
        gap = (best[0] + scores[0, 0]) - (best[1] + scores[0, 1])
        near += abs(gap) < 3e-7
        check_select(x, scores, 4, again=False)
        check_select(x, scores, 1, again=False)
    assert near > 30


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_beams_that_are_done_or_have_no_chance(dtype):
    import torch
    dt = getattr(torch, dtype)
    rng = np.random.default_rng(5)
    x = logits_like(rng, 12, 3001, dt)
    scores = rng.uniform(-8, -2, (3, 4))
    done = [1, 0, 0, 1, 0, 0, 0, 0, 1, 1, 1, 1]
    check_select(x, scores, 9, done, 77)                       # the last group: four candidates for nine places
    scores[1] = [-np.inf, -3, -np.inf, -np.inf]                # the first step
    check_select(x, scores, 9, done, 3000)
    scores[:] = -np.inf
    parent, token, score = check_select(x, scores, 9, done, 0)
    assert (parent == -1).all() and (token == -1).all() and (score == -np.inf).all()
    scores[:] = -1.0
    scores[2] = -1e30
    check_select(x, scores, 5, [1] * 12, 5)                    # ties of done beams
    # rows that are not read may hold anything
    y = x.clone()
    y[[0, 3, 8, 9, 10, 11]] = float("nan")
    scores = rng.uniform(-8, -2, (3, 4))
    check_select(y, scores, 9, done, 77)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_banned_tokens_and_numbers_that_are_none(dtype):
    import torch
    dt = getattr(torch, dtype)
    rng = np.random.default_rng(6)
    x = logits_like(rng, 6, 9001, dt)
    scores = rng.uniform(-8, -2, (2, 3))
    x[:, torch.tensor(rng.random(9001) < 0.9995, device="cuda")] = -float("inf")
    check_select(x, scores, 64)
    x[1] = -float("inf")
    check_select(x, scores, 128)
    x[0, 17], x[0, 4000], x[2, 9000] = float("nan"), float("inf"), float("nan")
    x[5] = float("nan")
    check_select(x, scores, 16, error=4)
    scores[0] = [np.nan, np.inf, -4.0]
    x = logits_like(rng, 6, 100, dt)
    check_select(x, scores, 5, error=4)
    low = torch.finfo(dt).min
    x = logits_like(rng, 6, 5000, dt)
    x[:, 1:4999] = low                                          # masked by the lowest number, not infinity
    x[3] = low                                                  # all of a row: as likely as one another
    check_select(x, rng.uniform(-8, -2, (2, 3)), 8)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_far_logits(dtype):
    """Past 2^20 in either direction, by themselves and beside ordinary rows."""
    import torch
    dt = getattr(torch, dtype)
    rng = np.random.default_rng(8)
    x = logits_like(rng, 12, 4099, torch.float32)
    x[0] += 3e6
    x[1] -= 3e6
    x[2] *= 1e9
    x[3, 7] = 2.0 ** 20 + 8
    x[4, 7] = -1e38
    x[5] = -3e38
    x[6] -= 1e5
    x[7] += 1000000
    x[8] = torch.finfo(dt).max
    check_select(x.to(dt), rng.uniform(-8, -2, (3, 4)), 30)
    check_select(x.to(dt), rng.uniform(-8, -2, (12, 1)), 30)


@pytest.mark.parametrize("offset", range(0, 9))
def test_rows_at_any_offset(offset):
    import torch
    rng = np.random.default_rng(offset)
    for dtype in (torch.float16, torch.bfloat16, torch.float32):
        store = torch.full((20000,), float("nan"), dtype=dtype, device="cuda")
        x = store[offset:offset + 6 * 3001].as_strided((6, 2999), (3001, 1))
        x.copy_(logits_like(rng, 6, 2999, dtype))
        check_select(x, rng.uniform(-8, -2, (2, 3)), 6)


def test_selections_in_graphs_and_on_streams():
    """Captured and replayed on new values, two calls at once on streams of their own."""
    import torch
    from paper_2608_28911_gb300 import semkv
    rng = np.random.default_rng(9)
    xs = [logits_like(rng, 8, 20001, torch.bfloat16) for _ in range(3)]
    scores = torch.tensor(rng.uniform(-3, -2, (2, 4)).astype(np.float32), device="cuda")

    def outs():
        return [torch.zeros((2, 6), dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]

    want = []
    for x in xs:
        o = outs()
        semkv.semkv_beam_select(x, scores, *o, semkv.beam_select_workspace(x, scores, 6))
        want.append(o)
    x, o = xs[0].clone(), outs()
    ws = semkv.beam_select_workspace(x, scores, 6)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        semkv.semkv_beam_select(x, scores, *o, ws)
    for i in (1, 2, 0):
        x.copy_(xs[i])
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(o, want[i]))
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [outs() for _ in xs]
    spaces = [semkv.beam_select_workspace(x, scores, 6) for x in xs]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, x, o, ws in zip(streams, xs, got, spaces):
            semkv.semkv_beam_select(x, scores, *o, ws, stream=s)
    torch.cuda.synchronize()
    for o, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(o, w))


@pytest.mark.parametrize("groups,beams", [(1, 4), (70, 5)])
def test_scores_in_place(groups, beams):
    """As many places as beams: the new scores may take the old ones' place."""
    import torch
    from paper_2608_28911_gb300 import semkv
    rng = np.random.default_rng(groups)
    x = logits_like(rng, groups * beams, 9001, torch.float16, 7)
    scores = torch.tensor(rng.uniform(-8, -2, (groups, beams)).astype(np.float32), device="cuda")
    want = check_select(x, scores.cpu().numpy(), beams)
    parent, token = [torch.empty((groups, beams), dtype=torch.int32, device="cuda") for _ in range(2)]
    semkv.semkv_beam_select(x, scores, parent, token, scores, semkv.beam_select_workspace(x, scores, beams))
    for a, b in zip((parent, token, scores), want):
        assert np.array_equal(a.cpu().numpy(), b)


# --------------------------------------------------------------------- reorder ------

def call_reorder(c, seqs, parent):
    from paper_2608_28911_gb300 import semkv
    ws = c.pages_workspace(len(parent), 0)
    ws.fill_(255)
    semkv.semkv_kv4_reorder(c, None if seqs is None else t32(seqs), t32(parent), ws)


MAPS = [([0, 1, 2, 3, 4], [0, 1, 2, 3, 4], 0), ([0, 1, 2, 3, 4], [1, 2, 3, 4, 0], 0), ([0, 1, 2, 3, 4], [2, 2, 2, 2, 2], 0),
        (None, [4, 3, -1, 1, 0], 0), ([3, 0], [1, 0], 0), ([2], [-1], 0), ([5, 6, 2, 3], [2, 3, 2, -1], 0), ([4, 1, 4, 0], [1, 0, 1, 2], 3),
        ([1, 9, 3, -1], [2, 0, 1, 2], 3), ([1, 3, 2], [1, 3, -2], 3), (None, [1, 0, 7, 2, -1, 6, 5, 0], 3), ([], [], 0)]


@pytest.mark.parametrize("P,wide", [(16, 0), (128, 0), (16, 9000), (32, 8190)])
@pytest.mark.parametrize("seqs,parent,error", MAPS)
def test_sequences_trade_places(P, wide, seqs, parent, error):
    """Cycles, copies, emptied ones, a list in its own order, and entries that are left out; tables that one kernel
    holds in its registers, and wider ones, which take two."""
    from paper_2608_28911_gb300 import semkv
    c = make([0, 1, 40, 300, 129], 1, 64, P, extra_seqs=2, spare=12, seed=P, more_pages=wide)
    plain = fill(c)
    call_reorder(c, seqs, parent)
    reorder(plain, seqs, parent)
    plain.same_state(c)
    assert int(c.dev_error.item()) == error
    # what comes after: new rows into pages that are shared now
    b = semkv.KV4Batch(7, cu=t32(range(8)), total=7, max_count=1)
    if not error:
        ws = c.pages_workspace(7)
        semkv.semkv_kv4_reserve(c, b, ws)
        want = plain.reserve(range(7), [1] * 7)
        if want is None:
            assert int(c.dev_error.item()) == 2
        else:
            assert b.start.tolist() == want
            plain.same_state(c)


@pytest.mark.parametrize("wide", [0, 300])
def test_a_search_over_many_sequences(wide):
    """300 branches of 20 prompts, several steps of random maps, one of them with a list entry twice."""
    rng = np.random.default_rng(4)
    lens = [int(x) for x in rng.integers(0, 200, 20)] + [0] * 280
    c = make(lens, 1, 64, 16, spare=0, seed=2, more_pages=wide)
    plain = fill(c)
    for step in range(6):
        n = int(rng.integers(1, 301))
        seqs = rng.permutation(300)[:n]
        parent = rng.integers(-1, n, n)
        if step == 3:
            seqs[n // 2] = seqs[0]
        call_reorder(c, seqs, parent)
        reorder(plain, seqs, parent)
        plain.same_state(c)
    assert (plain.refs >= 0).all() and plain.refs.sum() == sum(plain.used(t) for t in plain.length)


@pytest.mark.parametrize("wide", [0, 9000])
def test_reorders_in_a_graph(wide):
    import torch
    from paper_2608_28911_gb300 import semkv
    c = make([33, 70, 5, 100], 1, 64, 32, seed=1, more_pages=wide)
    plain = fill(c)
    seqs, parent, ws = t32([0, 1, 2, 3]), t32([0, 1, 2, 3]), c.pages_workspace(4, 0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        semkv.semkv_kv4_reorder(c, seqs, parent, ws)
    for p in ([1, 2, 3, 0], [1, 1, 0, 3], [0, 1, 2, 3], [3, -1, 3, 1]):
        parent.copy_(t32(p))
        g.replay()
        reorder(plain, [0, 1, 2, 3], p)
        plain.same_state(c)
    assert int(c.dev_error.item()) == 0


# -------------------------------------------------------------------- together ------

@pytest.mark.parametrize("dtype,P,pairs", [("bfloat16", 16, False), ("float16", 64, True)])
def test_a_search_as_it_is_run(dtype, P, pairs):
    """Three groups of four beams from prompts: reserve, rotated append, attention, logits, selection and
    reorder, each step's results against the definitions on what the GPU fed them."""
    import torch
    from paper_2608_28911_gb300 import semkv
    from test_gpu_kv4 import attend
    dt = getattr(torch, dtype)
    rng = np.random.default_rng(12)
    groups, beams, H, group, D, vocab, layers = 3, 4, 2, 3, 64, 701, 2
    n, Hq = groups * beams, H * group
    lens = [0] * n
    for g, t in enumerate((37, 5, 64)):
        lens[g * beams] = t
    c = make(lens, H, D, P, layers=layers, spare=60, seed=3, more_pages=3)
    plain = Plain(c)
    table = table_of(200, 32)
    rot = semkv.KV4Rotation(torch.tensor(table, device="cuda"), pairs)
    embed = torch.tensor(rng.standard_normal((vocab, H * (group + 2) * D)), dtype=dt, device="cuda")
    head = torch.tensor(rng.standard_normal((Hq * D, vocab)) * 0.1, dtype=dt, device="cuda")
    # prompts: rows behind the first beams of the groups
    first = t32([g * beams for g in range(groups)])
    counts = [lens[g * beams] for g in range(groups)]
    b = semkv.KV4Batch(groups, cu=cu_of(counts), seqs=first, start=t32([0] * groups), total=sum(counts), max_count=max(counts))
    x = embed[torch.tensor(rng.integers(0, vocab, sum(counts)), device="cuda")].view(sum(counts), -1, D)

    def write(b, x, rows):
        """rows: (sequence, position) of each."""
        for layer in range(layers):
            q, k, v = x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
            out = torch.empty((len(rows), Hq, D), dtype=dt, device="cuda")
            semkv.semkv_kv4_write_rotated(c, b, layer, rot, k, v, q, out)
            angles = table[[p for _, p in rows]]
            kf, vf = turn(k.float().cpu().numpy(), angles, 32, pairs), v.float().cpu().numpy()
            for i, (s, p) in enumerate(rows):
                plain.write(layer, s, p, kf[i], vf[i])
            assert torch.equal(out.cpu(), torch.tensor(turn(q.float().cpu().numpy(), angles, 32, pairs)).to(dt))
        return out

    write(b, x, [(g * beams, p) for g, t in enumerate(counts) for p in range(t)])
    # every beam begins as a branch of its group's first, which alone has a chance
    pages_ws = c.pages_workspace(n, 0)
    parent = [r // beams * beams for r in range(n)]
    semkv.semkv_kv4_reorder(c, None, t32(parent), pages_ws)
    reorder(plain, None, parent)
    scores = torch.full((groups, beams), -float("inf"), device="cuda")
    scores[:, 0] = 0
    done = torch.zeros((groups, beams), dtype=torch.bool, device="cuda")
    tokens = t32(rng.integers(0, vocab, n))
    out = [torch.empty((groups, beams), dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
    step = semkv.KV4Batch(n)
    for _ in range(9):
        semkv.semkv_kv4_reserve(c, step, pages_ws)
        want = plain.reserve(range(n), [1] * n)
        assert step.start.tolist() == want
        q = write(step, embed[tokens.long()].view(n, -1, D), list(zip(range(n), want)))
        same_pages_all(c, plain)
        y, _, _ = attend(c, plain, [1] * n, group, dt, q=q, with_cu=False, layer=1)
        logits = y.view(n, -1) @ head
        logits[:, 5] += 1.0                                     # the end token, likelier than the others
        semkv.semkv_beam_select(logits, scores, *out, semkv.beam_select_workspace(logits, scores, beams),
                                done=done, end_token=5, dev_error=c.dev_error)
        wp, wt, ws_ = select(logits.double().cpu().numpy(), scores.double().cpu().numpy(), beams, done.flatten().tolist(), 5)
        assert np.array_equal(out[0].cpu().numpy(), wp) and np.array_equal(out[1].cpu().numpy(), wt)
        assert (np.abs(out[2].cpu().numpy() - ws_) <= score_bound(vocab, ws_)).all()
        semkv.semkv_kv4_reorder(c, None, out[0].view(n), pages_ws)
        reorder(plain, None, wp.reshape(-1))
        plain.same_state(c, pages=False)
        tokens, scores = out[1].view(n).clone(), out[2].clone()
        done = tokens.view(groups, beams) == 5
    assert int(c.dev_error.item()) == 0 and bool(done.any())
    assert plain.refs.sum() == sum(plain.used(t) for t in plain.length)


def same_pages_all(c, plain):
    D, got = c.s.head_dim, c.pages.cpu().numpy()
    held = np.flatnonzero(plain.refs)
    assert np.array_equal(got[:, held][..., 16 * D:], plain.pages[:, held][..., 16 * D:])
    assert np.array_equal(bare(got[:, held], D), bare(plain.pages[:, held], D))
