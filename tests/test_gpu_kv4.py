"""The paged 4-bit cache on the GPU against its definition on the host (kv4_plain.py): stored bytes
and page states equal, attention within bounds derived from its roundings.  Pages start
filled with 0xFF (every scale a NaN), so whatever reads behind a sequence's end shows."""
import numpy as np
import pytest

from kv4_plain import Plain, attention_bounds, quantize, values

pytestmark = pytest.mark.gpu


def t32(x):
    import torch
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def cu_of(counts):
    return t32(np.concatenate([[0], np.cumsum(counts)]))


def make(lens, H=2, D=128, P=32, layers=1, spare=4, extra_seqs=0, scales=True, seed=0, more_pages=0):
    """A cache whose first sequences hold `lens` tokens (not written yet), pages in no order."""
    import torch
    from paper_2608_28911_gb300 import semkv
    rng = np.random.default_rng(seed)
    need = [-(-t // P) for t in lens]
    num = max(1, sum(need) + spare)
    width = max(need + [1]) + more_pages
    ks = vs = None
    if scales:
        ks = torch.tensor(rng.uniform(0.01, 0.03, (layers, H)).astype(np.float32), device="cuda")
        vs = torch.tensor(rng.uniform(0.001, 0.003, (layers, H)).astype(np.float32), device="cuda")
    c = semkv.KV4Cache(layers, H, D, P, num, len(lens) + extra_seqs, width, ks, vs)
    c.pages.fill_(255)
    order = rng.permutation(num)
    table, refs = c.table.cpu().numpy(), np.zeros(num, np.int32)
    at = 0
    for i, m in enumerate(need):
        table[i, :m] = order[at:at + m]
        refs[order[at:at + m]] = 1
        at += m
    c.table.copy_(t32(table))
    c.refs.copy_(t32(refs))
    c.length.copy_(t32(list(lens) + [0] * extra_seqs))
    return c


def rows_like(rng, shape, dtype):
    import torch
    x = rng.standard_normal(shape) * np.where(rng.random(shape[-1:]) < 0.05, 8, 1)
    return torch.tensor(x, dtype=dtype, device="cuda")


def fill(c, seed=1, layer=0, dtype=None):
    """Writes every token of every sequence by the framework; returns the host's cache."""
    import torch
    from paper_2608_28911_gb300 import semkv
    lens = c.length.cpu().numpy()
    rng = np.random.default_rng(seed)
    total, H, D = int(lens.sum()), c.s.kv_heads, c.s.head_dim
    if total:
        k, v = [rows_like(rng, (total, H, D), dtype or torch.float16) for _ in range(2)]
        b = semkv.KV4Batch(len(lens), cu=cu_of(lens), total=total, max_count=int(lens.max()))
        semkv.semkv_kv4_write(c, b, layer, k, v)
    return Plain(c)


# ------------------------------------------------------------- rows ------

SPECIAL = [0.0, -0.0, float("nan"), float("inf"), float("-inf"), 1e-7, -1e-7, 65504.0, -65504.0, 6e-8]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("D,P,H", [(128, 16, 3), (128, 64, 1), (64, 32, 2), (64, 128, 5)])
@pytest.mark.parametrize("scales", [True, False])
def test_rows_are_stored_as_defined_and_read_back(dtype, D, P, H, scales):
    import torch
    from paper_2608_28911_gb300 import semkv
    dt = getattr(torch, dtype)
    lens, counts = [0, 1, 40, 129, 16, 77], [0, 1, 7, 129, 16, 30]
    c = make(lens, H, D, P, layers=2, scales=scales, seed=D + P)
    plain = Plain(c)
    rng = np.random.default_rng(3)
    total = sum(counts) + 5                       # five rows that belong to nobody
    wide = rows_like(rng, (total, 2, H + 1, D), dt)   # K and V in one row, with something between
    wide[:, :, :, 5] = wide[:, :, :, 4] * 2.5        # values at and next to ties
    flat = wide.view(-1)
    flat[torch.tensor(rng.integers(0, flat.numel(), 60), device="cuda")] = \
        torch.tensor(SPECIAL * 6, dtype=dt, device="cuda")
    wide[3, :, :, 16:32] = 0
    wide[4, :, :, 0:16] = torch.tensor([i / 4 for i in range(16)], dtype=dt, device="cuda")   # exact ties
    k, v = wide[:, 0, :H], wide[:, 1, :H]
    seqs = [3, 1, 0, 5, 2, 4]                    # the list is in an order of its own
    counts = [counts[s] for s in seqs]
    start = [lens[s] - n for s, n in zip(seqs, counts)]
    start[1] = -1                                 # left out
    b = semkv.KV4Batch(6, cu=cu_of(counts), seqs=t32(seqs), start=t32(start), total=total, max_count=200)
    semkv.semkv_kv4_write(c, b, 1, k, v)
    kf, vf = k.float().cpu().numpy(), v.float().cpu().numpy()
    row = 0
    for s, n, p in zip(seqs, counts, start):
        for j in range(n if p >= 0 else 0):
            plain.write(1, s, p + j, kf[row + j], vf[row + j])
        row += n
    got = c.pages.cpu().numpy()
    # the sign of a zero code is the value's own: compared without it
    def bare(x):
        codes = x[..., :16 * D].copy()
        codes &= np.where(codes & 0x0F == 0x08, 0xF0, 0xFF).astype(np.uint8)
        codes &= np.where(codes & 0xF0 == 0x80, 0x0F, 0xFF).astype(np.uint8)
        return codes
    written = plain.pages != 255
    assert np.array_equal(got[..., 16 * D:], plain.pages[..., 16 * D:])
    same = bare(got) == bare(plain.pages)
    assert same.all(), np.argwhere(~same)[:5]
    assert np.array_equal(got[0], plain.pages[0]) and written.any()
    assert int(c.dev_error.item()) == 4            # the NaN and infinities were told of
    # and back
    c.dev_error.zero_()
    ko, vo = torch.full((total, H, D), 7.0, dtype=dt, device="cuda"), torch.full((total, H, D), 7.0, dtype=dt, device="cuda")
    semkv.semkv_kv4_read(c, b, 1, ko, vo)
    row = 0
    for s, n, p in zip(seqs, counts, start):
        for kv, out, g in ((0, ko, plain.kg[1]), (1, vo, plain.vg[1])):
            have = out[row:row + n].float().cpu().numpy()
            if p < 0:
                assert (have == 7).all()
                continue
            want = plain.rows(1, s, kv, range(p, p + n)).astype(np.float32) * g[:, None]
            want = torch.tensor(want).to(dt).float().numpy()
            assert np.array_equal(have, want)
        row += n
    assert (ko[row:] == 7).all() and (vo[row:] == 7).all()
    assert int(c.dev_error.item()) == 0


def test_rows_without_a_place_are_left_out():
    import torch
    from paper_2608_28911_gb300 import semkv
    c = make([40, 40, 40], H=1, D=64, P=16, spare=0)
    c.table[1, 1] = c.s.num_pages                # a page that is not there
    before = c.pages.clone()
    k = torch.ones((4, 1, 64), dtype=torch.float16, device="cuda")
    for seqs, start in (([7, -1, 3, 1], [0, 0, 0, 20]), ([0, 1, 2, 0], [48, 17, 1000, 2 ** 31 - 1])):
        c.dev_error.zero_()
        b = semkv.KV4Batch(4, seqs=t32(seqs), start=t32(start))
        semkv.semkv_kv4_write(c, b, 0, k, k)
        assert torch.equal(c.pages, before) and int(c.dev_error.item()) == 3
    c.dev_error.zero_()
    # ranges that are not: descending, past the rows, more than max_count
    for cu in ([0, 3, 2, 4, 4], [0, 0, 0, 0, 5], [-1, 0, 0, 0, 0], [4, 4, 4, 4, 4]):
        b = semkv.KV4Batch(4, cu=t32(cu), seqs=t32([0, 2, 0, 2]), start=t32([-1, 0, -1, -1]), total=4, max_count=1)
        semkv.semkv_kv4_write(c, b, 0, k, k)
        assert torch.equal(c.pages, before)


# -------------------------------------------------------- attention ------

def attend(c, plain, counts, group, dtype, window=0, seqs=None, seed=9, layer=0, with_cu=True, scale=None, q=None,
           lse=True):
    import torch
    from paper_2608_28911_gb300 import semkv
    H, D = c.s.kv_heads, c.s.head_dim
    n, total = len(counts), sum(counts) + (3 if with_cu else 0)
    scale = D ** -0.5 if scale is None else scale
    rng = np.random.default_rng(seed)
    if q is None:
        q = rows_like(rng, (total, H * group + 1, D), dtype)[:, :H * group]
    out = torch.full((total, H * group, D), 7.0, dtype=dtype, device="cuda")
    ls = torch.full((total, H * group), 7.0, device="cuda") if lse else None
    b = semkv.KV4Batch(n, cu=cu_of(counts) if with_cu else None, seqs=None if seqs is None else t32(seqs),
                       total=total, max_count=max(counts + [1]))
    ws = c.attention_workspace(b, H * group)
    ws.fill_(255)
    semkv.semkv_kv4_attention(c, b, layer, q, out, scale, ws, lse=ls, window=window)
    assert int(c.dev_error.item()) == 0
    row, worst = 0, 0.0
    qf, of = q.double().cpu().numpy(), out.double().cpu().numpy()
    lf = ls.double().cpu().numpy() if lse else None
    for i, m in enumerate(counts):
        s = i if seqs is None else seqs[i]
        want, wl, weight, size = plain.attend(layer, s, qf[row:row + m], scale, window)
        most = 2688 * float(plain.vg.max())
        tol, ltol = attention_bounds(want, wl, weight, size, dtype, D, max(1, int(plain.length[s])), most)
        off = np.abs(of[row:row + m] - want)
        assert (off <= tol).all(), (i, m, float((off / tol).max()))
        if lse:
            got = lf[row:row + m]
            assert np.array_equal(np.isinf(got), np.isinf(wl))
            fin = np.isfinite(wl)
            assert (np.abs(got[fin] - wl[fin]) <= ltol[fin]).all()
        if off.size:
            worst = max(worst, float((off / tol).max()))
        row += m
    assert (of[row:] == 7).all() and (not lse or (lf[row:] == 7).all())
    return out, ls, worst


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 64, 100, 500, 1000]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("group", [1, 4, 7])
def test_single_tokens(dtype, D, P, group):
    import torch
    c = make(LENS, 2, D, P, layers=2, seed=P)
    plain = fill(c, layer=1)
    attend(c, plain, [1] * len(LENS), group, getattr(torch, dtype), layer=1, with_cu=False)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("D,P", [(64, 16), (128, 32), (128, 128)])
@pytest.mark.parametrize("group,most", [(4, 2), (8, 2), (5, 5), (1, 40), (3, 70), (16, 20)])
@pytest.mark.parametrize("window", [0, 1, 37])
def test_several_tokens_some_without_a_past(dtype, D, P, group, most, window):
    import torch
    lens = [0, 1, 3, 33, 64, 200, 410]
    c = make(lens, 2, D, P, seed=most)
    plain = fill(c)
    seqs = [6, 0, 2, 5, 1, 4, 3]
    counts = [most, 1, min(most, 9), 0, most, 1, most]   # some have more rows than tokens
    attend(c, plain, counts, group, getattr(torch, dtype), window, seqs)


@pytest.mark.parametrize("window", [0, 3000])
def test_long_and_short_sequences_share_the_work(window):
    import torch
    lens = [20011, 3, 9000, 1, 5, 40000]
    c = make(lens, 1, 64, 64, seed=5)
    plain = fill(c)
    attend(c, plain, [1] * 6, 2, torch.float16, window)
    attend(c, plain, [5, 1, 0, 1, 2, 7], 2, torch.bfloat16, window)


@pytest.mark.parametrize("dtype,D,P,group", [("bfloat16", 128, 64, 4), ("float16", 64, 16, 2), ("float16", 128, 32, 3),
                                             ("bfloat16", 64, 128, 1)])
@pytest.mark.parametrize("window", [0, 200])
def test_prompts_and_chunks(dtype, D, P, group, window):
    """Many rows: tiles of 256 rows that several CTAs share, prompts, chunks behind a past, rows
    before the first token, and single tokens in the same call."""
    import torch
    lens = [640, 1, 900, 130, 257, 3000]
    c = make(lens, 1, D, P, seed=12)
    plain = fill(c)
    attend(c, plain, [640, 1, 300, 131, 0, 129], group, getattr(torch, dtype), window)


@pytest.mark.parametrize("group", [48, 256, 257, 300])
def test_large_groups(group):
    """A tile holds whole tokens: groups that leave rows of it empty, fill it, or do not fit one."""
    import torch
    c = make([200, 3, 70], 1, 64, 32, seed=3)
    plain = fill(c)
    attend(c, plain, [1, 3, 2], group, torch.float16)


@pytest.mark.parametrize("H,count", [(1, 8), (2, 12), (3, 40)])
def test_few_tiles_with_many_parts(H, count):
    """One long sequence whose few tiles are spread over all CTAs, the first rows of one without a past."""
    import torch
    c = make([9001, 5], H, 128, 32, seed=21)
    plain = fill(c)
    attend(c, plain, [count, 8], 8, torch.float16)


def test_many_sequences():
    import torch
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(0, 40, 700)]
    c = make(lens, 1, 64, 16, seed=6)
    plain = fill(c)
    attend(c, plain, [int(x) for x in rng.integers(0, 3, 700)], 2, torch.float16)


@pytest.mark.parametrize("group,counts", [(2, 1), (4, 20)])
def test_many_ragged_prompts_and_a_sequence_listed_twice(group, counts):
    """More sequences than a CTA has threads, in both kernels; some sequences are asked twice, and
    lse is left away."""
    import torch
    rng = np.random.default_rng(1)
    lens = [int(x) for x in rng.integers(0, 60, 1200)]
    c = make(lens, 1, 64, 16, seed=16)
    plain = fill(c)
    seqs = [int(x) for x in rng.integers(0, 1200, 1300)]
    attend(c, plain, [int(x) for x in rng.integers(0, counts + 1, 1300)], group, torch.bfloat16, seqs=seqs, lse=False)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 30, 128, 129])
def test_windows_at_the_ends_of_their_range(window):
    import torch
    c = make([700, 129, 1], 1, 64, 32, seed=17)
    plain = fill(c)
    attend(c, plain, [1, 2, 1], 3, torch.float16, window)
    attend(c, plain, [300, 129, 1], 3, torch.float16, window)


def test_two_calls_at_once():
    """Two streams, a workspace each, both kernels at work on one cache."""
    import torch
    from paper_2608_28911_gb300 import semkv
    lens = [4000, 900, 2500]
    c = make(lens, 2, 128, 64, seed=18)
    fill(c)
    calls = []
    for k, counts in enumerate(([1, 1, 1], [200, 64, 1], [3, 1, 2], [500, 1, 130])):
        rng = np.random.default_rng(k)
        q = rows_like(rng, (sum(counts), 8, 128), torch.float16)
        b = semkv.KV4Batch(3, cu=cu_of(counts), total=sum(counts), max_count=max(counts))
        calls.append((b, q, c.attention_workspace(b, 8)))
    def run(call, out):
        b, q, ws = call
        semkv.semkv_kv4_attention(c, b, 0, q, out, 128 ** -0.5, ws)
    alone = [torch.empty_like(q) for _, q, _ in calls]
    for call, out in zip(calls, alone):
        run(call, out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    outs = [[torch.empty_like(q) for _, q, _ in calls] for _ in range(5)]
    for row in outs:
        for s, call, out in zip(streams, calls, row):
            with torch.cuda.stream(s):
                run(call, out)
    torch.cuda.synchronize()
    for row in outs:
        for a, b in zip(alone, row):
            assert torch.equal(a, b)               # (the same split, the same order of sums)
    assert int(c.dev_error.item()) == 0


def test_large_and_small_logits():
    """Weights far apart, all equal, and logits whose size makes the reference exponent move often."""
    import torch
    lens = [300, 300, 300]
    c = make(lens, 2, 128, 32, seed=8)
    plain = fill(c)
    for scale in (0.0, 1.0, -0.3):
        attend(c, plain, [1, 2, 3], 4, torch.float16, scale=scale)
    rng = np.random.default_rng(4)
    for size in (1e-30, 1e30, 1e-4):
        q = (rows_like(rng, (9, 8, 128), torch.float32) * size).bfloat16()
        attend(c, plain, [1, 2, 3], 4, torch.bfloat16, scale=0.1 / size, q=q)


def test_rows_with_nan_stay_alone():
    import torch
    c = make([100, 50], 1, 128, 32, seed=8)
    plain = fill(c)
    from paper_2608_28911_gb300 import semkv
    rng = np.random.default_rng(4)
    q = rows_like(rng, (4, 4, 128), torch.float16)
    clean, _, _ = attend(c, plain, [3, 1], 4, torch.float16, q=torch.cat([q, q[:3]]))
    bad = q.clone()
    bad[1, 2, 5] = float("nan")
    out = torch.empty_like(bad)
    b = semkv.KV4Batch(2, cu=cu_of([3, 1]), total=4, max_count=3)
    semkv.semkv_kv4_attention(c, b, 0, bad, out, 128 ** -0.5, c.attention_workspace(b, 4))
    assert out[1, 2].isnan().all()
    keep = torch.ones((4, 4), dtype=torch.bool)
    keep[1, 2] = False
    assert torch.equal(out[keep.cuda()], clean[:4][keep.cuda()])


def test_attention_with_wrong_indices_reports_them():
    import torch
    from paper_2608_28911_gb300 import semkv
    c = make([50, 60], 1, 64, 16)
    fill(c)
    q = torch.ones((3, 2, 64), dtype=torch.float16, device="cuda")
    for seqs, cu in (([0, 5], [0, 1, 2]), ([-1, 0], [0, 1, 2]), ([0, 1], [0, 1, 4]), ([0, 1], [0, 3, 3])):
        c.dev_error.zero_()
        out = torch.full_like(q, 7.0)
        b = semkv.KV4Batch(2, cu=t32(cu), seqs=t32(seqs), total=3, max_count=2)
        semkv.semkv_kv4_attention(c, b, 0, q, out, 0.1, c.attention_workspace(b, 2))
        assert int(c.dev_error.item()) == 3 and (out[2] == 7).all()
    c.table[0, 2] = c.s.num_pages + 3            # read as page 0
    c.dev_error.zero_()
    b = semkv.KV4Batch(2)
    out = torch.full_like(q[:2], 7.0)
    semkv.semkv_kv4_attention(c, b, 0, q[:2], out, 0.1, c.attention_workspace(b, 2))
    assert int(c.dev_error.item()) == 3


def test_cache_past_32_bit_offsets():
    """A pool of more than 4 GB with the pages of a sequence at both ends."""
    import torch
    from paper_2608_28911_gb300 import semkv
    H, D, P = 8, 128, 128
    num = (5 << 30) // (H * P * 18 * D // 16)
    c = semkv.KV4Cache(1, H, D, P, num, 1, 3)
    c.table.copy_(t32([[num - 1, 0, num - 2]]))
    c.length.copy_(t32([300]))
    c.refs[t32([0, num - 1, num - 2]).long()] = 1
    rng = np.random.default_rng(1)
    k, v = [rows_like(rng, (300, H, D), torch.float16) for _ in range(2)]
    b = semkv.KV4Batch(1, cu=cu_of([300]), total=300, max_count=300)
    semkv.semkv_kv4_write(c, b, 0, k, v)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    semkv.semkv_kv4_read(c, b, 0, ko, vo)
    for x, back in ((k, ko), (v, vo)):
        want = values(*quantize(x.float().cpu().numpy(), np.ones((300, H), np.float32)))
        assert np.array_equal(back.double().cpu().numpy(), want)      # (exact in fp16: g is 1)
    q = rows_like(rng, (1, H, D), torch.float16)
    out = torch.empty_like(q)
    b1 = semkv.KV4Batch(1)
    semkv.semkv_kv4_attention(c, b1, 0, q, out, D ** -0.5, c.attention_workspace(b1, H))
    p = torch.softmax(torch.einsum("hd,thd->ht", q[0].double(), ko.double()) * D ** -0.5, -1)
    want = torch.einsum("ht,thd->hd", p, vo.double())
    assert float((out[0] - want).abs().max()) < 4e-3  # (weights and result in fp16, values below 4)
    assert int(c.dev_error.item()) == 0


# ------------------------------------------------------------ pages ------

def pages_ws(c, n, tokens=-1):
    ws = c.pages_workspace(n, tokens)
    ws.fill_(255)
    return ws


@pytest.mark.parametrize("D,P,H", [(128, 16, 3), (64, 128, 1), (128, 64, 2)])
def test_fork_reserve_free_follow_the_definition(D, P, H):
    import torch
    from paper_2608_28911_gb300 import semkv
    rng = np.random.default_rng(P)
    c = make([2 * P + 5, 3 * P, 0, 7], H, D, P, layers=3, spare=60, extra_seqs=12, more_pages=4, seed=2)
    c.pages.copy_(torch.randint(0, 256, c.pages.shape, dtype=torch.uint8))
    plain = Plain(c)
    for step in range(25):
        kind = rng.integers(0, 3)
        ids = rng.permutation(16)
        if kind == 0:
            n = int(rng.integers(1, 5))
            src, dst = ids[:n], ids[4:4 + n]
            if step % 3 == 0:
                src = np.full(n, src[0])
            semkv.semkv_kv4_fork(c, t32(src), t32(dst))
            plain.fork(src.tolist(), dst.tolist())
        elif kind == 1:
            n = int(rng.integers(1, 4))
            seqs = np.concatenate([ids[:n], ids[:1]])     # one is listed twice
            semkv.semkv_kv4_free(c, t32(seqs))
            plain.free(seqs.tolist())
        else:
            n = int(rng.integers(1, 8))
            counts = rng.integers(0, 2 * P if step % 2 else 3, n)
            cu = cu_of(counts)
            start = t32(np.full(n, -7))
            b = semkv.KV4Batch(n, cu=cu, seqs=t32(ids[:n]), start=start, total=int(counts.sum()), max_count=2 * P)
            c.dev_error.zero_()
            semkv.semkv_kv4_reserve(c, b, pages_ws(c, n))
            want = plain.reserve(ids[:n].tolist(), counts.tolist())
            assert np.array_equal(start.cpu().numpy(), [-1] * n if want is None else want)
            assert int(c.dev_error.item()) == (2 if want is None else 0)
        plain.same_state(c)
    semkv.semkv_kv4_free(c, t32(range(16)))
    assert int(c.refs.abs().sum().item()) == 0 and int(c.length.sum().item()) == 0


def test_reserve_over_many_sequences_and_pages():
    import torch
    from paper_2608_28911_gb300 import semkv
    rng = np.random.default_rng(1)
    n, num = 2500, 30001
    c = semkv.KV4Cache(1, 1, 64, 16, num, n, 40)
    held = rng.random(num) < 0.2
    c.refs.copy_(t32(held))
    plain = Plain(c)
    counts = rng.integers(0, 150, n)
    order = rng.permutation(n)
    for _ in range(2):
        b = semkv.KV4Batch(n, cu=cu_of(counts), seqs=t32(order), total=int(counts.sum()), max_count=150)
        semkv.semkv_kv4_reserve(c, b, pages_ws(c, n))
        want = plain.reserve(order.tolist(), counts.tolist())    # (the second time the pool is too small)
        assert np.array_equal(b.start.cpu().numpy(), [-1] * n if want is None else want)
        assert int(c.dev_error.item()) == (2 if want is None else 0)
        plain.same_state(c, pages=False)


def test_reserve_refuses_whole():
    from paper_2608_28911_gb300 import semkv
    c = make([20, 30], 1, 64, 16, spare=3, extra_seqs=1)
    plain = Plain(c)
    for counts in ([30, 30, 30], [1, 1, 100]):         # too few pages, a table too short
        b = semkv.KV4Batch(3, cu=cu_of(counts), total=sum(counts), max_count=100)
        c.dev_error.zero_()
        semkv.semkv_kv4_reserve(c, b, pages_ws(c, 3))
        assert b.start.tolist() == [-1] * 3 and int(c.dev_error.item()) == 2
        plain.same_state(c)
    c.dev_error.zero_()
    b = semkv.KV4Batch(4, seqs=t32([1, 5, 1, -2]))       # out of range, twice
    semkv.semkv_kv4_reserve(c, b, pages_ws(c, 4))
    assert b.start.tolist() == [30, -1, -1, -1] and int(c.dev_error.item()) == 3
    assert plain.reserve([1, 5, 1, -2], [1] * 4) == [30, -1, -1, -1]
    plain.same_state(c)


def test_fork_leaves_out_what_it_may_not_do():
    from paper_2608_28911_gb300 import semkv
    c = make([20, 30], 1, 64, 16, extra_seqs=4)
    plain = Plain(c)
    for src, dst, error in (([0], [1], 2), ([0, 1], [2, 2], 3), ([0, 2], [2, 3], 3), ([0, 9], [9, 2], 3),
                            ([0, 1, 0], [3, 4, 5], 0)):
        c.dev_error.zero_()
        semkv.semkv_kv4_fork(c, t32(src), t32(dst))
        plain.fork(src, dst)
        assert int(c.dev_error.item()) == error, (src, dst)
        plain.same_state(c)


@pytest.mark.parametrize("D,P,H", [(128, 16, 3), (64, 128, 1), (128, 64, 2)])
def test_compact_follows_the_definition(D, P, H):
    import torch
    from paper_2608_28911_gb300 import semkv
    lens = [5 * P + 3, 0, 3 * P, 1, 2 * P + 9]
    c = make(lens, H, D, P, layers=2, spare=14, extra_seqs=2, seed=4)
    c.pages.copy_(torch.randint(0, 256, c.pages.shape, dtype=torch.uint8))
    semkv.semkv_kv4_fork(c, t32([0, 2]), t32([5, 6]))
    plain = Plain(c)
    rng = np.random.default_rng(2)
    for seqs, T, rate in (([5], 5 * P + 3, 0.3), ([0, 6, 1, 0], 2 * P + 1, 0.5), ([4, 9], 3 * P, 0.0), ([2, 3], 0, 0.0)):
        keep = (rng.random((len(seqs), T)) < rate).astype(np.uint8) * rng.integers(1, 256, (len(seqs), T)).astype(np.uint8)
        c.dev_error.zero_()
        semkv.semkv_kv4_compact(c, t32(seqs), torch.tensor(keep, device="cuda"), pages_ws(c, len(seqs), T))
        assert plain.compact(seqs, keep)
        assert int(c.dev_error.item()) == (3 if len(set(seqs)) < len(seqs) or 9 in seqs else 0)
        plain.same_state(c)


def test_compact_refuses_whole():
    import torch
    from paper_2608_28911_gb300 import semkv
    c = make([100, 100], 1, 64, 16, spare=5)
    plain = Plain(c)
    keep = torch.ones((2, 100), dtype=torch.uint8, device="cuda")
    semkv.semkv_kv4_compact(c, t32([0, 1]), keep, pages_ws(c, 2, 100))
    assert int(c.dev_error.item()) == 2
    plain.same_state(c)


def test_compact_of_a_long_sequence():
    import torch
    from paper_2608_28911_gb300 import semkv
    T = 40003
    c = make([T], 1, 64, 64, spare=700, seed=4)
    c.pages.copy_(torch.randint(0, 256, c.pages.shape, dtype=torch.uint8))
    plain = Plain(c)
    keep = (np.random.default_rng(3).random((1, T)) < 0.6).astype(np.uint8)
    semkv.semkv_kv4_compact(c, t32([0]), torch.tensor(keep, device="cuda"), pages_ws(c, 1, T))
    assert plain.compact([0], keep)
    plain.same_state(c)


# --------------------------------------------------------- together ------

@pytest.mark.parametrize("graph", [False, True])
def test_a_served_batch(graph):
    """Prompts, branches, tokens, pruning by the framework's own selection, attention after each,
    on a stream of its own; the token steps also from a captured graph, replayed."""
    import torch
    from paper_2608_28911_gb300 import semkv
    H, G, D, P, layers = 2, 4, 128, 32, 2
    c = make([0, 0], H, D, P, layers=layers, spare=90, extra_seqs=6, more_pages=12)
    rng = np.random.default_rng(11)
    plain = Plain(c)

    def run_step(b, k, v, q, out, lse, pws, aws):
        semkv.semkv_kv4_reserve(c, b, pws)
        for layer in range(layers):
            semkv.semkv_kv4_write(c, b, layer, k[layer], v[layer])
            semkv.semkv_kv4_attention(c, b, layer, q[layer], out[layer], D ** -0.5, aws, lse=lse[layer])

    def check(seqs, counts, k, v, q, out, lse):
        start = plain.reserve(seqs, counts)
        row = 0
        kf, vf, qf = [x.double().cpu().numpy() for x in (k, v, q)]
        for s, m, p in zip(seqs, counts, start):
            for layer in range(layers):
                for j in range(m):
                    plain.write(layer, s, p + j, kf[layer, row + j].astype(np.float32), vf[layer, row + j].astype(np.float32))
            row += m
        row = 0
        for s, m in zip(seqs, counts):
            for layer in range(layers):
                want, wl, weight, size = plain.attend(layer, s, qf[layer, row:row + m], D ** -0.5)
                tol, ltol = attention_bounds(want, wl, weight, size, out.dtype, D, int(plain.length[s]), 2688 * float(plain.vg.max()))
                assert (np.abs(out[layer, row:row + m].double().cpu().numpy() - want) <= tol).all()
                assert (np.abs(lse[layer, row:row + m].double().cpu().numpy() - wl) <= ltol).all()
            row += m
        assert np.array_equal(plain.length, c.length.cpu().numpy()) and np.array_equal(plain.refs, c.refs.cpu().numpy())

    def tensors(total):
        k, v = [rows_like(rng, (layers, total, H, D), torch.bfloat16) for _ in range(2)]
        q = rows_like(rng, (layers, total, H * G, D), torch.bfloat16)
        return k, v, q, torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")

    def step(seqs, counts, replays=1):
        total = sum(counts)
        b = semkv.KV4Batch(len(seqs), cu=cu_of(counts), seqs=t32(seqs), total=total, max_count=max(counts))
        pws, aws = c.pages_workspace(len(seqs)), c.attention_workspace(b, H * G)
        t = tensors(total)
        if not graph:
            run_step(b, *t, pws, aws)
            check(seqs, counts, *t)
            return
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run_step(b, *t, pws, aws)
        for _ in range(replays):
            new = tensors(total)
            for a, x in zip(t[:3], new[:3]):
                a.copy_(x)
            g.replay()
            check(seqs, counts, *t)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        stream.wait_stream(torch.cuda.default_stream())
        step([0, 1], [70, 41])
        semkv.semkv_kv4_fork(c, t32([0, 0, 1]), t32([2, 3, 4]))
        plain.fork([0, 0, 1], [2, 3, 4])
        step([0, 2, 3, 1, 4], [1] * 5, replays=3)
        semkv.semkv_kv4_free(c, t32([2]))
        plain.free([2])
        # pruned to the tokens that the framework's selection keeps
        T = int(plain.length[3])
        scores = torch.tensor(rng.random((1, T)).astype(np.float32), device="cuda")
        keep, slot = torch.empty((1, T), dtype=torch.uint8, device="cuda"), torch.empty((1, T), dtype=torch.int32, device="cuda")
        semkv.semkv_rank_assign(scores, T // 2, keep, slot)
        semkv.semkv_kv4_compact(c, t32([3]), keep, c.pages_workspace(1, T))
        assert plain.compact([3], keep.cpu().numpy())
        step([3, 0, 4], [3, 1, 2], replays=2)
        assert int(c.dev_error.item()) == 0
    torch.cuda.synchronize()


def test_pages_become_rows_for_the_packed_pools():
    """A finished prompt leaves the paged cache for the mixed-precision pools: read back, ranked,
    quantized and packed as any prompt."""
    import torch
    from paper_2608_28911_gb300 import semkv
    T, H = 333, 2
    c = make([T], H, 128, 64)
    fill(c)
    b = semkv.KV4Batch(1, cu=cu_of([T]), total=T, max_count=T)
    k, v = [torch.empty((T, H, 128), dtype=torch.float16, device="cuda") for _ in range(2)]
    semkv.semkv_kv4_read(c, b, 0, k, v)
    k5, v5 = [x.permute(1, 0, 2).contiguous().view(1, 1, H, T, 128) for x in (k, v)]
    scores = torch.empty((1, T), device="cuda")
    semkv.semkv_score_kv_norm(v5, scores)
    desc = semkv.QuantDesc(semkv.BASE_AFFINE, 8, 8)
    pool = semkv.KVCache(desc, 1, 1, H, 4 * H, hi_cap=T, lo_cap=16)
    is_high, slot = torch.empty((1, T), dtype=torch.uint8, device="cuda"), torch.empty((1, T), dtype=torch.int32, device="cuda")
    semkv.semkv_rank_assign(scores, T, is_high, slot)
    semkv.semkv_quantize_pack(desc, k5, v5, is_high, slot, T, pool)
    import oracle
    from paper_2608_28911_gb300 import synthetic
    oc = oracle.Cache(base=0, L_hi=8, L_lo=8, batch=1, layers=1, kv_heads=H, q_heads=4 * H, block=128,
                      hi_cap=pool.s.hi_cap, lo_cap=pool.s.lo_cap)
    bits = [synthetic.f16_bits(x.cpu().numpy()) for x in (k5, v5)]
    oracle.quantize_prompt(oc, *bits, scores.cpu().numpy(), 1, 1)
    assert np.array_equal(pool.hi_pool.cpu().numpy()[..., :T, :], oc.hi_pool[..., :T, :])
    # the rows are the cache's: each value its code times scale times 1, exact in fp16 but for the heads' scales
    plain = Plain(c)
    for x, kv, g in ((k, 0, plain.kg), (v, 1, plain.vg)):
        want = plain.rows(0, 0, kv, range(T)).astype(np.float32) * g[0][:, None]
        assert np.array_equal(x.cpu().numpy(), want.astype(np.float16))
