"""CPU checks of the paged 4-bit cache's entry points: sizes, and what they refuse before
anything is launched.  No kernel runs; the pointers are never followed."""
import ctypes

import numpy as np
import pytest
import torch

from kv4_plain import E4M3, LEVELS, nearest, quantize, values

FAKE = 1 << 20
EINVAL, EALIGN, EUNSUPPORTED, EWORKSPACE = 1, 2, 4, 6


@pytest.fixture(scope="module")
def sk():
    from paper_2608_28911_gb300 import build
    build.build()
    from paper_2608_28911_gb300 import semkv
    return semkv


def cache(sk, **kw):
    f = dict(layers=2, kv_heads=2, head_dim=128, page_tokens=64, num_pages=10, max_seqs=4, max_pages=3, pages=FAKE,
             k_scale=None, v_scale=None, table=FAKE, length=FAKE, refs=FAKE, dev_error=FAKE)
    f.update(kw)
    return sk.KV4CacheStruct(**f)


def batch(sk, **kw):
    f = dict(n=2, total=2, max_count=1, seqs=None, cu=None, start=FAKE)
    f.update(kw)
    return sk.KV4BatchStruct(**f)


def calls(sk, c, b, layer=0, dtype=0, stride=256, x=FAKE, ws=FAKE, q_heads=8, q_stride=1024, window=0, lse=None):
    """Every entry point's status for one cache and batch, whose work is refused in each."""
    L, r, p = sk.LIB, ctypes.byref, (lambda s: None if s is None else ctypes.byref(s))
    del r
    return {
        "reserve": L.semkv_kv4_reserve(p(c), p(b), ws, 0, None),
        "write": L.semkv_kv4_write(p(c), p(b), layer, dtype, x, stride, x, stride, None),
        "read": L.semkv_kv4_read(p(c), p(b), layer, dtype, x, x, None),
        "attention": L.semkv_kv4_attention(p(c), p(b), layer, dtype, x, q_stride, q_heads, x, lse, 1.0, window, ws, 0, None),
        "fork": L.semkv_kv4_fork(p(c), 0 if b is None else b.n, FAKE, FAKE, None),
        "free": L.semkv_kv4_free(p(c), 0 if b is None else b.n, FAKE, None),
        "compact": L.semkv_kv4_compact(p(c), 0 if b is None else b.n, FAKE, FAKE, 5, ws, 0, None),
    }


def test_tile_and_workspace_sizes(sk):
    assert sk.semkv_kv4_tile_bytes(128) == 2304 and sk.semkv_kv4_tile_bytes(64) == 1152
    assert sk.semkv_kv4_tile_bytes(96) == 0 and sk.semkv_kv4_tile_bytes(0) == 0
    c = cache(sk)
    size = sk.LIB.semkv_kv4_pages_workspace_bytes(ctypes.byref(c), 2, 0)
    assert size >= 4 * (4 + 3 + 2 + 4 + 10) and size % 16 == 0
    assert sk.LIB.semkv_kv4_pages_workspace_bytes(ctypes.byref(c), 2, 1000) >= size + 8000
    assert sk.LIB.semkv_kv4_pages_workspace_bytes(ctypes.byref(cache(sk, head_dim=100)), 2, 0) == 0
    assert sk.LIB.semkv_kv4_pages_workspace_bytes(ctypes.byref(c), -1, 0) == 0
    assert 4 * (4 + 3 + 2 + 4 + 10) <= sk.LIB.semkv_kv4_pages_workspace_bytes(ctypes.byref(c), 2, -1) < size


@pytest.mark.parametrize("field,bad,status", [
    ("layers", 0, EINVAL), ("kv_heads", 0, EINVAL), ("num_pages", 0, EINVAL), ("max_seqs", 0, EINVAL),
    ("max_pages", 0, EINVAL), ("head_dim", 96, EUNSUPPORTED), ("head_dim", 256, EUNSUPPORTED),
    ("page_tokens", 8, EUNSUPPORTED), ("page_tokens", 48, EUNSUPPORTED), ("page_tokens", 256, EUNSUPPORTED),
    ("max_pages", 1 << 25, EUNSUPPORTED), ("pages", None, EINVAL), ("table", None, EINVAL), ("length", None, EINVAL),
    ("refs", None, EINVAL), ("pages", FAKE + 8, EALIGN), ("refs", FAKE + 4, EALIGN), ("table", FAKE + 2, EALIGN),
    ("k_scale", FAKE + 1, EALIGN)])
def test_caches_that_are_refused(sk, field, bad, status):
    got = calls(sk, cache(sk, **{field: bad}), batch(sk))
    assert set(got.values()) == {status}, got


def test_no_cache_no_batch(sk):
    assert set(calls(sk, None, batch(sk)).values()) == {EINVAL}
    got = calls(sk, cache(sk), None)
    assert [got[k] for k in ("reserve", "write", "read", "attention")] == [EINVAL] * 4


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), EINVAL), (dict(total=-1), EINVAL), (dict(max_count=0), EINVAL), (dict(total=1), EINVAL),
    (dict(n=65536, total=65536), EUNSUPPORTED), (dict(seqs=FAKE + 2), EALIGN), (dict(cu=FAKE + 2), EALIGN)])
def test_batches_that_are_refused(sk, kw, status):
    got = calls(sk, cache(sk), batch(sk, **kw))
    assert [got[k] for k in ("reserve", "write", "read", "attention")] == [status] * 4, got


def test_arguments_that_are_refused(sk):
    c, b = cache(sk), batch(sk)
    no_start = calls(sk, c, batch(sk, start=None))
    assert [no_start[k] for k in ("reserve", "write", "read")] == [EINVAL] * 3
    for kw, status, names in (
            (dict(layer=2), EINVAL, ("write", "read", "attention")),
            (dict(layer=-1), EINVAL, ("write", "read", "attention")),
            (dict(dtype=2), EUNSUPPORTED, ("write", "read", "attention")),
            (dict(x=None), EINVAL, ("write", "read", "attention")),
            (dict(x=FAKE + 8), EALIGN, ("write", "read", "attention")),
            (dict(stride=255), EINVAL, ("write",)), (dict(stride=260), EALIGN, ("write",)),
            (dict(q_heads=0), EINVAL, ("attention",)), (dict(q_heads=7), EINVAL, ("attention",)),
            (dict(q_stride=1000), EINVAL, ("attention",)), (dict(q_stride=1028), EALIGN, ("attention",)),
            (dict(window=-1), EINVAL, ("attention",)), (dict(lse=FAKE + 2), EALIGN, ("attention",))):
        got = calls(sk, c, b, **{"ws": FAKE, **kw})
        for n in names:
            assert got[n] == status, (kw, n, got)
    big = batch(sk, cu=FAKE, max_count=1 << 29)
    assert calls(sk, c, big)["attention"] == EUNSUPPORTED
    # workspaces: none, too small, misaligned
    got = calls(sk, c, b, ws=None)
    assert got["reserve"] == EWORKSPACE and got["compact"] == EWORKSPACE
    size = sk.LIB.semkv_kv4_pages_workspace_bytes(ctypes.byref(c), 2, -1)
    assert sk.LIB.semkv_kv4_reserve(ctypes.byref(c), ctypes.byref(b), FAKE, size - 1, None) == EWORKSPACE
    assert sk.LIB.semkv_kv4_reserve(ctypes.byref(c), ctypes.byref(b), FAKE + 8, size, None) == EWORKSPACE
    assert sk.LIB.semkv_kv4_compact(ctypes.byref(c), 2, None, None, 5, FAKE, 1 << 30, None) == EINVAL
    assert sk.LIB.semkv_kv4_compact(ctypes.byref(c), 2, None, FAKE, -1, FAKE, 1 << 30, None) == EINVAL
    assert sk.LIB.semkv_kv4_fork(ctypes.byref(c), 2, None, FAKE, None) == EINVAL


def test_empty_calls_are_nothing(sk):
    c, b = cache(sk), batch(sk, n=0, total=0)
    got = calls(sk, c, b)
    assert set(got.values()) == {0}, got
    assert sk.LIB.semkv_kv4_write(ctypes.byref(c), ctypes.byref(batch(sk, cu=FAKE, total=0)), 0, 0, FAKE, 256, FAKE, 256, None) == 0


def test_empty_tensors_have_no_address(sk):
    c = cache(sk)
    for b in (batch(sk, n=0, total=0, max_count=0, start=None), batch(sk, cu=FAKE, total=0, max_count=0),
              batch(sk, n=0, total=0, cu=FAKE, start=None)):
        got = calls(sk, c, b, x=None)
        assert [got[k] for k in ("write", "read", "attention")] == [0] * 3, got
        assert b.n > 0 or got["reserve"] == 0
    assert calls(sk, c, batch(sk, n=0, total=0), layer=2)["write"] == EINVAL


def test_steps_of_too_many_rows_are_refused(sk):
    got = calls(sk, cache(sk), batch(sk, cu=FAKE, total=(1 << 30) + 1))
    assert [got[k] for k in ("reserve", "write", "read", "attention")] == [EUNSUPPORTED] * 4, got


def test_the_binding_refuses_tensors_that_do_not_fit(sk):
    cpu = dict(device="cpu")
    with pytest.raises(ValueError):
        sk.KV4Cache(1, 1, 96, 16, 4, 1, 1, **cpu)
    c = sk.KV4Cache(1, 2, 64, 16, 4, 1, 1, **cpu)
    with pytest.raises(ValueError):
        sk.KV4Cache.over(c.pages, c.table, c.length, c.refs[:3], 64)
    with pytest.raises(ValueError):
        sk.KV4Cache.over(c.pages, c.table, c.length, c.refs, 128)
    with pytest.raises(ValueError):
        sk.KV4Cache.over(c.pages, c.table.long(), c.length, c.refs, 64)
    with pytest.raises(ValueError):
        sk.KV4Cache.over(c.pages, c.table, c.length, c.refs, 64, k_scale=torch.ones(2))
    assert sk.KV4Cache.over(c.pages, c.table, c.length, c.refs, 64, k_scale=torch.ones(1, 2)).s.page_tokens == 16
    x = torch.zeros((3, 2, 64), dtype=torch.float16)
    for bad in (x[:2], x[:, :1], x[..., :32], x.transpose(0, 1).contiguous().transpose(0, 1)):
        with pytest.raises(ValueError):
            sk._rows(bad, "k", 3, 2, 64)
    assert sk._rows(x, "k", 3, 2, 64) == 128
    for a, b in ((x.float(), x.float()), (x, x.bfloat16())):
        with pytest.raises(ValueError):
            sk._type16(a, b, "k and v")
    assert sk._type16(x, x, "k") == 0 and sk._type16(x.bfloat16(), x.bfloat16(), "k") == 1
    wide = torch.zeros((3, 5, 64), dtype=torch.bfloat16)
    assert sk._rows(wide[:, 1:3], "k", 3, 2, 64) == 320


# ------------------------------------------------- the plain form's own pins ------

def test_plain_formats_are_the_numbers_they_should_be():
    t = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(E4M3, t)
    x = np.random.default_rng(0).uniform(0, 460, 20000)
    x = np.concatenate([x, (E4M3[:-1] + E4M3[1:]) / 2, 2.0 ** np.arange(-14.0, 9)])
    want = torch.tensor(np.minimum(x, 448)).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(nearest(E4M3, np.minimum(x, 448).astype(np.float32)), want)
    assert list(nearest(LEVELS, [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 9])) == [0, 2, 2, 4, 4, 6, 6, 7]


def test_plain_quantizer_is_within_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((500, 64)).astype(np.float32)
    c, s = quantize(x, np.full(500, 0.004, np.float32))
    v = values(c, s) * 0.004
    scale = np.repeat(E4M3[s] * 0.004, 16, -1)
    # a scale is at most 1/16 below the largest's sixth; a value at most half the widest step off
    assert (np.abs(v - x) <= np.where(np.abs(x) <= 6 * scale, 1.0, 0.4) * scale * (1 + 1e-6)).all()
