"""The paged 4-bit cache on the GPU where its format and its softmax have their ends."""
import numpy as np
import pytest

from kv4_plain import Plain
from test_gpu_kv4 import attend, cu_of, fill, make, rows_like, t32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("D", [64, 128])
def test_blocks_without_a_scale_hold_zeros(dtype, D):
    """Where the block's scale is 0 every code is 0, the sign bit too, and what is read back is +0."""
    import torch
    from paper_2608_28911_gb300 import semkv
    dt = getattr(torch, dtype)
    c = make([40], 2, D, 16, scales=False)
    plain = Plain(c)
    rng = np.random.default_rng(D)
    # a sixth of the largest is below 2^-10, half of the smallest scale
    x = [torch.tensor(rng.uniform(-0.0058, 0.0058, (40, 2, D)), dtype=dt, device="cuda") for _ in range(2)]
    for y in x:
        y[3] = -0.0
        y[4, :, 3] = float("nan")
        y[5, :, :16] = -1.0                          # beside a block that has a scale
    b = semkv.KV4Batch(1, cu=cu_of([40]), total=40, max_count=40)
    semkv.semkv_kv4_write(c, b, 0, *x)
    back = [torch.full_like(y, 7.0) for y in x]
    semkv.semkv_kv4_read(c, b, 0, *back)
    for j in range(40):
        plain.write(0, 0, j, *[y[j].float().cpu().numpy() for y in x])
    assert (plain.pages[..., :16 * D] == 0).any()
    assert np.array_equal(c.pages.cpu().numpy(), plain.pages)
    for y in back:
        bits = y.view(torch.int16)
        bits[5, :, :16] = 0
        assert not bits.any()


@pytest.mark.parametrize("count", [2, 8, 25, 75])    # 8 rows, a tile of 32, halves of a block, two blocks
@pytest.mark.parametrize("dtype,power", [("float16", 20), ("float16", 24), ("float16", 27), ("float16", 30), ("float16", 60), ("float16", 117),
                                         ("bfloat16", 22), ("bfloat16", 26), ("bfloat16", 30), ("bfloat16", 90), ("bfloat16", 100), ("bfloat16", 120)])
@pytest.mark.parametrize("sign", [1, -1])
def test_logits_of_any_finite_size(count, dtype, power, sign):
    """Logits of about +-2^power.  A row that sees one token returns it, equal logits share the weight, a logit that
    is twice the others' takes all of it or none, whatever the size.

    Every q and every K entry is one power of two or the same number, so equal logits are equal bit by bit and
    their weights are one number w; w is rounded to fp16 (2^-11), the products' sums lose 17 addends' last places for
    each 16 tokens.  lse goes through fewer than eight roundings of binary32."""
    import torch
    from paper_2608_28911_gb300 import semkv
    dt, D, H, G = getattr(torch, dtype), 128, 2, 4
    lens, counts, special = [1, 100, 300], [1, count, count], 137
    c = make(lens, H, D, 32, seed=4, scales=False)
    rng = np.random.default_rng(1)
    v = rows_like(rng, (sum(lens), H, D), torch.float16)
    k = torch.ones_like(v)
    k[1 + 100 + special] *= 2                     # the block's scale doubles, the codes are the same
    semkv.semkv_kv4_write(c, semkv.KV4Batch(3, cu=cu_of(lens), total=sum(lens), max_count=300), 0, k, v)
    plain = Plain(c)
    e = 10 if dtype == "float16" else power - 4   # 128 dims times D^-0.5 are about 2^3.5
    scale = 2.0 ** (power - 17) if dtype == "float16" else D ** -0.5
    total = sum(counts)
    q = torch.full((total, H * G, D), sign * 2.0 ** e, dtype=dt, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((total, H * G), 7.0, device="cuda")
    b = semkv.KV4Batch(3, cu=cu_of(counts), total=total, max_count=max(counts))
    semkv.semkv_kv4_attention(c, b, 0, q, out, scale, c.attention_workspace(b, H * G), lse=lse)
    assert int(c.dev_error.item()) == 0
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    u = torch.finfo(dt).eps / 2
    row = 0
    for s, m in enumerate(counts):
        ks, vs = [plain.rows(0, s, kv, range(lens[s])) for kv in (0, 1)]
        one = ks[0, 0].sum() * sign * 2.0 ** e * float(np.float32(scale))
        for j in range(m):
            seen = np.arange(lens[s] - m + j + 1)
            if s == 2:
                seen = seen[seen == special] if sign > 0 else seen[seen != special]
            want, size = vs[seen].mean(0), np.abs(vs[seen]).mean(0)        # [H][D]
            tol = u * np.abs(want) + (1 + u) * (2.0 ** -10 + 17 * 2.0 ** -23 * np.ceil(lens[s] / 16)) * size + 2.0 ** -25
            off = np.abs(got[row + j].reshape(H, G, D) - want[:, None])
            assert (off <= tol[:, None]).all(), (s, j, float(np.nanmax(off)))
            l = (2 * one if s == 2 and sign > 0 else one) + np.log(len(seen))
            assert (np.abs(gl[row + j] - l) <= abs(l) * 2.0 ** -21 + 2.0 ** -18).all(), (s, j, gl[row + j], l)
        row += m


def test_a_step_that_names_no_largest_count():
    """Without max_count every sequence may have as many rows as the step: none is left out."""
    import torch
    from paper_2608_28911_gb300 import semkv
    c = make([60, 9, 30], 2, 64, 16, spare=9, more_pages=1)
    plain = fill(c)
    counts = [5, 0, 12]
    b = semkv.KV4Batch(3, cu=cu_of(counts), total=17)
    q = rows_like(np.random.default_rng(3), (17, 4, 64), torch.float16)
    out = torch.full_like(q, 7.0)
    semkv.semkv_kv4_attention(c, b, 0, q, out, 0.125, c.attention_workspace(b, 4))
    assert int(c.dev_error.item()) == 0
    want, _, _ = attend(c, plain, counts, 2, torch.float16, q=torch.cat([q, q[:3]]), scale=0.125)
    assert (out - want[:17]).abs().max() < 0.01 and not (out == 7).any()
    semkv.semkv_kv4_reserve(c, b, c.pages_workspace(3))
    assert b.start.tolist() == [60, 9, 30] and c.length.tolist() == [65, 9, 42]
    assert semkv.KV4Batch(5).s.max_count == 1      # one row to a sequence


def test_page_calls_over_many_sequences():
    """More sequences than a plan has threads, forked, freed and pruned in one call each."""
    import torch
    from paper_2608_28911_gb300 import semkv
    rng = np.random.default_rng(2)
    n, T = 1500, 70
    lens = [int(x) for x in rng.integers(0, T, n)] + [4000]
    c = make(lens, 1, 64, 16, spare=6000, extra_seqs=n, seed=3)
    c.pages.copy_(torch.randint(0, 256, c.pages.shape, dtype=torch.uint8))
    plain = Plain(c)
    src, dst = rng.integers(0, n + 1, n), n + 1 + rng.permutation(n)
    semkv.semkv_kv4_fork(c, t32(src), t32(dst))
    plain.fork(src.tolist(), dst.tolist())
    plain.same_state(c)
    gone = rng.permutation(2 * n + 1)[:n]
    semkv.semkv_kv4_free(c, t32(gone))
    plain.free(gone.tolist())
    plain.same_state(c)
    seqs = rng.permutation(2 * n + 1)[:n + 200]
    keep = (rng.random((len(seqs), T)) < 0.4).astype(np.uint8)
    semkv.semkv_kv4_compact(c, t32(seqs), torch.tensor(keep, device="cuda"), c.pages_workspace(len(seqs), T))
    assert plain.compact(seqs.tolist(), keep)
    plain.same_state(c)
    assert int(c.dev_error.item()) == 0
