"""Attention over the paged 4-bit cache with much work for each worker: ranges of more than 64 units, rings and
buffers that turn many times, several long items one behind the other on one CTA; and the many-row kernel at the
ends of its inputs.  Attention may list a sequence as often as it likes, so a few sequences of some thousand tokens,
listed in no order, are work enough; the definition is evaluated once for each."""
import numpy as np
import pytest

from kv4_plain import Plain, attention_bounds
from test_gpu_kv4 import cu_of, fill, make, rows_like, t32

pytestmark = pytest.mark.gpu


def sms():
    import torch
    return torch.cuda.get_device_properties(0).multi_processor_count


def marked(c, seed=2):
    """Writes rows of the usual kind for K; V is 0 but for one dim, which names the tile of 16 tokens, so that a
    tile dropped, repeated or taken from elsewhere moves results by a good part of themselves."""
    import torch
    from paper_2608_28911_gb300 import semkv
    lens, H, D = c.length.cpu().numpy(), c.s.kv_heads, c.s.head_dim
    total = int(lens.sum())
    k = rows_like(np.random.default_rng(seed), (total, H, D), torch.float16)
    v = torch.zeros_like(k)
    pos = torch.cat([torch.arange(int(t)) + 5000 * i for i, t in enumerate(lens)]).cuda()
    for h in range(H):
        dim = (pos // 16 * 5 + 11 * h) % D
        v[torch.arange(total, device="cuda"), h, dim] = 1 + (pos // 16 % 3).half()
    b = semkv.KV4Batch(len(lens), cu=cu_of(lens), total=total, max_count=int(lens.max()))
    semkv.semkv_kv4_write(c, b, 0, k, v)
    return Plain(c)


def define(plain, seq, q, scale, window):
    """One sequence's rows q [m][Hq][D] by the definition in 64 bits: out, lse, weight, size as Plain.attend has them,
    the host's decoded rows multiplied on the GPU."""
    import torch
    m, Hq, D = q.shape
    G, t = Hq // plain.H, int(plain.length[seq])
    k, v = [torch.tensor(plain.rows(0, seq, kv, range(t)), device="cuda").transpose(0, 1) for kv in (0, 1)]   # [H][t][D]
    kg, vg = [torch.tensor(g[0], device="cuda").double().view(-1, 1, 1) for g in (plain.kg, plain.vg)]
    x = q.double().view(m, plain.H, G, D).permute(1, 2, 0, 3).reshape(plain.H, G * m, D)
    p = (t - m + torch.arange(m, device="cuda")).repeat(G)[:, None]
    at = torch.arange(t, device="cuda")
    see = (at <= p) & ((at > p - window) if window else (at >= 0))
    z = (x @ k.transpose(1, 2) * (scale * kg)).masked_fill(~see, -float("inf"))
    size = (x.abs() @ k.abs().transpose(1, 2) * (abs(scale) * kg)).masked_fill(~see, 0).amax(-1)
    lse = torch.logsumexp(z, -1)
    w = torch.where(see.any(-1)[:, None], torch.softmax(z, -1), torch.zeros_like(z))
    back = lambda y: y.reshape(plain.H, G, m, *y.shape[2:]).movedim(2, 0).reshape(m, Hq, *y.shape[2:]).cpu().numpy()
    return back(w @ v * vg), back(lse), back(w @ v.abs() * vg), back(size)


def bounds(got, dtype, D, tokens, longest, v_most):
    """Tolerances as attention_bounds has them, but with the sums' length that of the longest range of one worker,
    not of the sequence.  The parts of a row, at most one for each such range and one at either end, are joined behind
    that: each costs a product, an addition and an approximate power of two in both sums, together less than 2^-20."""
    tol, ltol = attention_bounds(*got, dtype, D, min(tokens, longest), v_most)
    parts = tokens / longest + 2
    return tol + parts * 2.0 ** -20 * got[2] + max(0, tokens - longest) * 2.0 ** -33 * v_most, ltol + parts * 2.0 ** -20


def check(c, plain, listing, counts, group, dtype, window, longest, scale=None, q_sets=None, repeat=True):
    """The sequences of `listing`, each with counts[seq] rows of its own query set, in one call, against the definition."""
    import torch
    from paper_2608_28911_gb300 import semkv
    H, D = c.s.kv_heads, c.s.head_dim
    scale = D ** -0.5 if scale is None else scale
    rng = np.random.default_rng(5)
    if q_sets is None:
        q_sets = [rows_like(rng, (m, H * group, D), dtype) for m in counts]
    q = torch.cat([q_sets[s] for s in listing])
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    per = [counts[s] for s in listing]
    b = semkv.KV4Batch(len(listing), cu=cu_of(per), seqs=t32(listing), total=sum(per), max_count=max(counts))
    ws = c.attention_workspace(b, H * group)
    ws.fill_(255)
    semkv.semkv_kv4_attention(c, b, 0, q, out, scale, ws, lse=lse, window=window)
    assert int(c.dev_error.item()) == 0
    if repeat:
        out2, lse2 = torch.full_like(q, 7.0), torch.full_like(lse, 7.0)
        semkv.semkv_kv4_attention(c, b, 0, q, out2, scale, ws, lse=lse2, window=window)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
    starts = np.concatenate([[0], np.cumsum(per)])
    worst = 0.0
    for s, m in enumerate(counts):
        want = define(plain, s, q_sets[s], scale, window)
        tol, ltol = bounds(want, dtype, D, int(plain.length[s]), longest, 2688 * float(plain.vg.max()))
        w, l, tol, ltol = [torch.tensor(x, device="cuda") for x in (want[0], want[1], tol, ltol)]
        for i in np.flatnonzero(np.asarray(listing) == s):
            rows = slice(int(starts[i]), int(starts[i + 1]))
            off = (out[rows].double() - w).abs()
            assert (off <= tol).all(), (i, s, float((off / tol).max()))
            seen = l > -float("inf")
            assert torch.equal(seen, lse[rows] > -float("inf"))
            assert ((lse[rows].double() - l).abs()[seen] <= ltol[seen]).all(), (i, s)
            worst = max(worst, float((off / tol).max()))
    return worst


@pytest.mark.parametrize("dtype,D,P,group,count", [("bfloat16", 128, 16, 4, 1), ("float16", 64, 64, 4, 2), ("float16", 128, 64, 6, 2),
                                                   ("bfloat16", 128, 64, 4, 5), ("bfloat16", 64, 16, 8, 4)])
@pytest.mark.parametrize("window", [0, 1500])
def test_few_rows_with_long_ranges(dtype, D, P, group, count, window):
    """A warp with more than 64 units: its page numbers are fetched anew inside an item, its ring turns twenty times."""
    import torch
    H, lens = 2, [4000, 2777, 1503]
    c = make(lens, H, D, P, seed=P)
    plain = marked(c)
    workers = sms() * (16 if group * count <= 8 else 8)
    units = [(min(t, window + count - 1 if window else t)) // 32 for t in lens]      # (or one or two more)
    n = int(72 * workers / (H * (np.mean(units) + 2))) + 1
    listing = np.random.default_rng(0).integers(0, 3, n)
    work = sum(H * (units[s] + 4) for s in listing)
    assert H * sum(units[s] + 2 for s in listing) / workers > 64
    check(c, plain, listing, [count] * 3, group, getattr(torch, dtype), window, 32 * (work // workers + 1))


@pytest.mark.parametrize("dtype,D,P,group,count", [("bfloat16", 128, 64, 4, 160), ("float16", 64, 16, 2, 300), ("float16", 128, 16, 8, 33),
                                                   ("bfloat16", 128, 32, 4, 30), ("float16", 64, 128, 8, 5)])
@pytest.mark.parametrize("window", [0, 1500])
def test_many_rows_with_long_ranges(dtype, D, P, group, count, window):
    """A CTA with several items of more than eight units, of two blocks and of one, one behind the other."""
    import torch
    H, lens = 2, [2900, 1501, 2222]
    c = make(lens, H, D, P, seed=P)
    plain = marked(c)
    tokens = 256 // group
    tiles = -(-count // tokens)
    n = 5 * sms() // (H * tiles) + 1
    listing = np.random.default_rng(0).integers(0, 3, n)
    work = sum(H * tiles * (min(lens[s] + tokens, window + tokens if window else 1 << 30) + 448) for s in listing)
    check(c, plain, listing, [count] * 3, group, getattr(torch, dtype), window, work // sms() + 256)


def test_one_long_sequence_with_marked_values():
    """40000 tokens over all workers: a dropped or repeated tile of 16 shows, and sums are no longer than a range."""
    import torch
    c = make([40000], 1, 64, 64, seed=5)
    plain = marked(c)
    for count in (1, 9):                            # (few units: no range is shorter than four, so none longer than five)
        check(c, plain, [0], [count], 2, torch.float16, 0, 5 * 32)
    check(c, plain, [0], [200], 2, torch.bfloat16, 0, 2 * (40000 + 600) // sms() + 256)


# ------------------------------------------- many rows at the ends of their inputs ------

ROWS = [(4, 12), (4, 30), (4, 80)]   # group and tokens: 48 and 120 rows (halves of a block in turn), 320 (two blocks)


@pytest.mark.parametrize("group,count", ROWS)
def test_many_rows_with_large_and_small_logits(group, count):
    """Scale 0 and below 0, and bf16 rows whose sizes need the whole range of the factor, rows of different sizes side
    by side and items of different sizes one behind the other."""
    import torch
    lens = [300, 700, 500]
    c = make(lens, 2, 128, 32, seed=8)
    plain = fill(c)
    listing = list(np.random.default_rng(0).integers(0, 3, 3 * sms() // 2))
    for dtype in (torch.float16, torch.bfloat16):
        for scale in (0.0, 1.0, -0.3):
            check(c, plain, listing, [count] * 3, group, dtype, 0, 4000, scale=scale)
    rng = np.random.default_rng(4)
    for size in (1e-30, 1e30, 1e-4):
        sets = [(rows_like(rng, (count, 2 * group, 128), torch.float32) * size).bfloat16() for _ in range(3)]
        for sign in (1, -1):
            check(c, plain, listing, [count] * 3, group, torch.bfloat16, 0, 4000, scale=sign * 0.1 / size, q_sets=sets)
    # powers of two from row to row: a factor that went to another row or item would be off by them
    power = torch.tensor(2.0 ** rng.integers(-6, 7, (3, count, 2 * group, 1)), device="cuda", dtype=torch.float32)
    sets = [(rows_like(rng, (count, 2 * group, 128), torch.float32) * power[s] * 0.1).bfloat16() for s in range(3)]
    check(c, plain, listing, [count] * 3, group, torch.bfloat16, 0, 4000, q_sets=sets)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("group,count", ROWS)
def test_many_rows_with_nan_stay_alone(dtype, group, count):
    import torch
    from paper_2608_28911_gb300 import semkv
    c = make([400, 150], 1, 128, 32, seed=8)
    fill(c)
    rng = np.random.default_rng(4)
    q = rows_like(rng, (count + 50, group, 128), getattr(torch, dtype))
    b = semkv.KV4Batch(2, cu=cu_of([count, 50]), total=count + 50, max_count=max(count, 50))
    bad = q.clone()
    bad[1, 2, 5] = float("nan")
    got = []
    for x in (q, bad):
        out, lse = torch.empty_like(x), torch.empty(x.shape[:2], device="cuda")
        semkv.semkv_kv4_attention(c, b, 0, x, out, 128 ** -0.5, c.attention_workspace(b, group), lse=lse)
        got.append((out, lse))
    assert got[1][0][1, 2].isnan().all() and got[1][1][1, 2].isnan()
    keep = torch.ones((count + 50, group), dtype=torch.bool, device="cuda")
    keep[1, 2] = False
    assert torch.equal(got[0][0][keep], got[1][0][keep]) and torch.equal(got[0][1][keep], got[1][1][keep])


@pytest.mark.parametrize("group,count", ROWS)
def test_many_rows_with_wrong_indices(group, count):
    """A sequence out of range or with a wrong row range is left out, its rows as they were, and the others are right."""
    import torch
    from paper_2608_28911_gb300 import semkv
    c = make([300, 260, 90], 2, 64, 16)
    plain = fill(c)
    rng = np.random.default_rng(7)
    total = 3 * count
    q = rows_like(rng, (total, 2 * group, 64), torch.float16)
    good = [0, count, 2 * count, 3 * count]
    for seqs, cu, wrong in (([0, 7, 2], good, [1]), ([-1, 1, 0], good, [0]), ([0, 1, 2], [0, count, 2 * count, total + 1], [2]),
                            ([0, 1, 2], [0, 2 * count, 2 * count, 3 * count], [0]), ([9, 1, 2], [0, count, count - 1, 2 * count - 1], [0, 1])):
        c.dev_error.zero_()
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        b = semkv.KV4Batch(3, cu=t32(cu), seqs=t32(seqs), total=total, max_count=count)
        semkv.semkv_kv4_attention(c, b, 0, q, out, 0.125, c.attention_workspace(b, 2 * group), lse=lse)
        assert int(c.dev_error.item()) == 3
        touched = torch.zeros(total, dtype=torch.bool, device="cuda")
        for i in range(3):
            if i in wrong or cu[i + 1] == cu[i]:
                continue
            rows = slice(cu[i], cu[i + 1])
            want = define(plain, seqs[i], q[rows], 0.125, 0)
            tol, ltol = bounds(want, torch.float16, 64, 300, 1 << 20, 2688 * float(plain.vg.max()))
            assert (np.abs(out[rows].double().cpu().numpy() - want[0]) <= tol).all()
            seen = np.isfinite(want[1])
            assert (np.abs(lse[rows].double().cpu().numpy() - want[1])[seen] <= ltol[seen]).all()
            touched[rows] = True
        assert (out[~touched] == 7).all() and (lse[~touched] == 7).all()
    # a page that is not there is read as page 0: the sequence's rows are some numbers, the others' are right
    c.table[0, 2] = c.s.num_pages + 3
    c.dev_error.zero_()
    out = torch.full_like(q, 7.0)
    b = semkv.KV4Batch(3, cu=t32(good), total=total, max_count=count)
    semkv.semkv_kv4_attention(c, b, 0, q, out, 0.125, c.attention_workspace(b, 2 * group))
    assert int(c.dev_error.item()) == 3
    for i in (1, 2):
        want = define(plain, i, q[i * count:(i + 1) * count], 0.125, 0)
        tol, _ = bounds(want, torch.float16, 64, 300, 1 << 20, 2688 * float(plain.vg.max()))
        assert (np.abs(out[i * count:(i + 1) * count].double().cpu().numpy() - want[0]) <= tol).all()


@pytest.mark.parametrize("count", [40, 200])
def test_many_rows_past_32_bit_offsets(count):
    import torch
    from paper_2608_28911_gb300 import semkv
    H, D, P = 8, 128, 128
    num = (5 << 30) // (H * P * 18 * D // 16)
    c = semkv.KV4Cache(1, H, D, P, num, 1, 3)
    c.table.copy_(t32([[num - 1, 0, num - 2]]))
    c.length.copy_(t32([300]))
    rng = np.random.default_rng(1)
    k, v = [rows_like(rng, (300, H, D), torch.float16) for _ in range(2)]
    semkv.semkv_kv4_write(c, semkv.KV4Batch(1, cu=cu_of([300]), total=300, max_count=300), 0, k, v)
    small = make([300], H, D, P, scales=False)          # the same rows in a small pool
    semkv.semkv_kv4_write(small, semkv.KV4Batch(1, cu=cu_of([300]), total=300, max_count=300), 0, k, v)
    q = rows_like(rng, (count, H, D), torch.float16)
    b = semkv.KV4Batch(1, cu=cu_of([count]), total=count, max_count=count)
    got = []
    for x in (c, small):
        got.append(torch.empty_like(q))
        semkv.semkv_kv4_attention(x, b, 0, q, got[-1], D ** -0.5, x.attention_workspace(b, H))
    assert torch.equal(*got) and int(c.dev_error.item()) == 0
    want = define(Plain(small), 0, q, D ** -0.5, 0)
    tol, _ = bounds(want, torch.float16, D, 300, 1 << 20, 2688)
    assert (np.abs(got[0].double().cpu().numpy() - want[0]) <= tol).all()
