"""CPU checks of a search step's entry points (rotated write, beam selection, reorder): sizes, and what the
library and the binding refuse before anything is launched.  No kernel runs; the pointers are never followed."""
import ctypes

import numpy as np
import pytest
import torch

from search_plain import select, table_of, turn
from test_kv4_abi import EALIGN, EINVAL, EUNSUPPORTED, EWORKSPACE, FAKE, batch, cache, sk  # noqa: F401


# ------------------------------------------------------------- rotated write ------

def rotated(sk, c=None, b=None, layer=0, r=None, positions=None, dtype=0, q=FAKE, qs=1024, heads=8, qo=FAKE, qos=1024,
            k=FAKE, ks=256, v=FAKE, vs=256, **kw):
    f = dict(rot_dim=128, layout=0, rows=10, cos_sin=FAKE)
    f.update(kw)
    r = sk.KV4RotationStruct(**f) if r is None else r
    c = cache(sk) if c is None else c
    b = batch(sk) if b is None else b
    p = (lambda s: ctypes.byref(s) if s else None)
    return sk.LIB.semkv_kv4_write_rotated(p(c), p(b), layer, p(r), positions, dtype, q, qs, heads, qo, qos, k, ks, v, vs, None)


@pytest.mark.parametrize("kw,status", [
    (dict(c=False), EINVAL), (dict(b=False), EINVAL), (dict(r=False), EINVAL), (dict(layer=2), EINVAL), (dict(layer=-1), EINVAL),
    (dict(rot_dim=0), EINVAL), (dict(rot_dim=144), EINVAL), (dict(rot_dim=-16), EINVAL), (dict(rot_dim=24), EUNSUPPORTED),
    (dict(layout=2), EUNSUPPORTED), (dict(rows=0), EINVAL), (dict(cos_sin=None), EINVAL), (dict(cos_sin=FAKE + 4), EALIGN),
    (dict(positions=FAKE + 2), EALIGN), (dict(dtype=2), EUNSUPPORTED), (dict(dtype=-1), EUNSUPPORTED),
    (dict(q=None), EINVAL), (dict(qo=None), EINVAL), (dict(heads=-1), EINVAL), (dict(qs=1023), EINVAL), (dict(qos=1016), EINVAL),
    (dict(qs=1028), EALIGN), (dict(qos=1028), EALIGN), (dict(q=FAKE + 8), EALIGN), (dict(qo=FAKE + 2), EALIGN),
    (dict(qos=2048), EINVAL), (dict(heads=(1 << 23) + 1, qs=1 << 31, qos=1 << 31), EUNSUPPORTED), (dict(k=None), EINVAL),
    (dict(v=None), EINVAL), (dict(k=FAKE + 8), EALIGN), (dict(v=FAKE + 8), EALIGN), (dict(ks=255), EINVAL),
    (dict(vs=260), EALIGN)])
def test_rotated_writes_that_are_refused(sk, kw, status):
    assert rotated(sk, **kw) == status


def test_rotated_writes_go_by_what_every_call_refuses(sk):
    assert rotated(sk, c=cache(sk, head_dim=96)) == EUNSUPPORTED
    assert rotated(sk, c=cache(sk, pages=FAKE + 8)) == EALIGN
    assert rotated(sk, b=batch(sk, start=None)) == EINVAL
    assert rotated(sk, b=batch(sk, total=1)) == EINVAL
    assert rotated(sk, c=cache(sk, head_dim=64), rot_dim=80) == EINVAL


def test_rotated_writes_of_nothing(sk):
    none = batch(sk, n=0, total=0, start=None)
    assert rotated(sk, b=none) == 0
    assert rotated(sk, b=none, q=None, qo=None, k=None, v=None) == 0
    assert rotated(sk, b=none, heads=0, q=None, qo=None, qs=0, qos=0) == 0
    assert rotated(sk, b=batch(sk, cu=FAKE, total=0)) == 0
    assert rotated(sk, b=none, layer=2) == EINVAL


# ------------------------------------------------------------------- reorder ------

def test_reorders_that_are_refused(sk):
    c = cache(sk)
    size = sk.LIB.semkv_kv4_pages_workspace_bytes(ctypes.byref(c), 2, 0)

    def call(c=c, n=2, seqs=FAKE, parent=FAKE, ws=FAKE, size=size):
        return sk.LIB.semkv_kv4_reorder(ctypes.byref(c) if c else None, n, seqs, parent, ws, size, None)

    for kw, status in ((dict(c=None), EINVAL), (dict(c=cache(sk, refs=None)), EINVAL), (dict(n=-1), EINVAL), (dict(n=65536), EUNSUPPORTED),
                       (dict(seqs=FAKE + 2), EALIGN), (dict(parent=None), EINVAL), (dict(parent=FAKE + 1), EALIGN),
                       (dict(ws=None), EWORKSPACE), (dict(ws=FAKE + 8), EWORKSPACE), (dict(size=size - 1), EWORKSPACE),
                       (dict(n=3), EWORKSPACE), (dict(n=0, seqs=None, parent=None, ws=None, size=0), 0)):
        assert call(**kw) == status, kw


# ------------------------------------------------------------ beam selection ------

def beam(sk, groups=3, beams=4, vocab=1000, dtype=0, logits=FAKE, stride=1000, scores=FAKE, done=None, end=0, k=8, parent=FAKE,
         token=FAKE, score=FAKE, err=None, ws=FAKE, size=1 << 30):
    return sk.LIB.semkv_beam_select(groups, beams, vocab, dtype, logits, stride, scores, done, end, k, parent, token, score, err, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(groups=-1), EINVAL), (dict(beams=0), EINVAL), (dict(beams=129), EUNSUPPORTED), (dict(k=0), EINVAL), (dict(k=129), EUNSUPPORTED),
    (dict(vocab=0), EINVAL), (dict(vocab=(1 << 24) + 1, stride=1 << 25), EUNSUPPORTED), (dict(groups=1 << 18, beams=5), EUNSUPPORTED),
    (dict(dtype=3), EUNSUPPORTED), (dict(dtype=-1), EUNSUPPORTED), (dict(stride=999), EINVAL), (dict(stride=0), EINVAL),
    (dict(logits=None), EINVAL), (dict(scores=None), EINVAL), (dict(parent=None), EINVAL), (dict(token=None), EINVAL),
    (dict(score=None), EINVAL), (dict(logits=FAKE + 1), EALIGN), (dict(dtype=2, logits=FAKE + 2), EALIGN), (dict(scores=FAKE + 2), EALIGN),
    (dict(parent=FAKE + 2), EALIGN), (dict(token=FAKE + 1), EALIGN), (dict(score=FAKE + 2), EALIGN), (dict(err=FAKE + 2), EALIGN),
    (dict(done=FAKE, end=-1), EINVAL), (dict(done=FAKE, end=1000), EINVAL), (dict(ws=None), EWORKSPACE), (dict(ws=FAKE + 4), EWORKSPACE),
    (dict(groups=0), 0), (dict(groups=0, logits=None, scores=None, parent=None, token=None, score=None, ws=None, size=0), 0)])
def test_beam_selections_that_are_refused(sk, kw, status):
    assert beam(sk, **kw) == status


def test_beam_workspaces(sk):
    size = sk.semkv_beam_select_workspace_bytes
    want = size(3, 4, 1000, torch.float16, 8)
    assert want >= 12 * (16 + 24 * 8) and want % 16 == 0
    assert beam(sk, size=want - 1) == EWORKSPACE
    assert size(0, 4, 1000, torch.float16, 8) == 0 and size(3, 200, 1000, torch.float16, 8) == 0
    assert size(64, 16, 131072, torch.bfloat16, 32) >= size(64, 16, 131072, torch.bfloat16, 16) > 0
    with pytest.raises(ValueError):
        size(3, 4, 1000, torch.float64, 8)
    assert size(1 << 20, 1, 1 << 24, torch.float32, 128) >= (1 << 20) * 144 * 8


# ---------------------------------------------------------------- the binding ------

@pytest.fixture()
def here(sk, monkeypatch):  # noqa: F811
    monkeypatch.setattr(sk, "_raw_device", lambda: -1)       # where CPU tensors are
    monkeypatch.setattr(sk, "_stream", lambda stream: None)
    return sk


def test_the_binding_refuses_rotations_that_do_not_fit(here):
    c = here.KV4Cache(1, 2, 64, 16, 4, 2, 1, device="cpu")
    i32 = dict(dtype=torch.int32)
    b = here.KV4Batch(2, cu=torch.zeros(3, **i32), start=torch.zeros(2, **i32), total=0, max_count=1)
    x, q = torch.zeros((0, 2, 64), dtype=torch.float16), torch.zeros((0, 4, 64), dtype=torch.float16)
    for bad in (torch.zeros((4, 24)), torch.zeros((4, 32), dtype=torch.float64), torch.zeros(32), torch.zeros((0, 32)), torch.zeros((4, 64))[:, :32],
                torch.zeros(4 * 32 + 1)[1:].view(4, 32)):
        with pytest.raises(ValueError, match="cos_sin"):
            here.KV4Rotation(bad)
    r = here.KV4Rotation(torch.zeros((4, 32)), pairs=True)
    assert (r.s.rot_dim, r.s.layout, r.s.rows) == (32, 1, 4) and here.KV4Rotation(torch.zeros((4, 32))).s.layout == 0
    here.semkv_kv4_write_rotated(c, b, 0, r, x, x)
    here.semkv_kv4_write_rotated(c, b, 0, r, x, x, q, q, positions=torch.zeros(0, **i32))
    for args, kw in (((x, x, q), {}), ((x, x), dict(q_out=q)), ((x, x, q, q.bfloat16()), {}), ((x, x, q.bfloat16(), q.bfloat16()), {}),
                     ((x, x, q[:, 0], q[:, 0]), {}), ((x, x, q, x), {}), ((x, x.bfloat16()), {}), ((x[:, :1], x), {}),
                     ((x, x), dict(positions=torch.zeros(1, **i32))), ((x, x), dict(positions=torch.zeros(0, dtype=torch.int64)))):
        with pytest.raises(ValueError):
            here.semkv_kv4_write_rotated(c, b, 0, r, *args, **kw)
    with pytest.raises(here.SemkvError):
        here.semkv_kv4_write_rotated(c, b, 0, here.KV4Rotation(torch.zeros((4, 128))), x, x)   # more dims than a head has
    monkey = here._raw_device
    try:
        here._raw_device = lambda: 3
        with pytest.raises(ValueError, match="current CUDA device"):
            here.semkv_kv4_write_rotated(c, b, 0, r, x, x)
    finally:
        here._raw_device = monkey


def test_the_binding_refuses_selections_that_do_not_fit(here):
    x, s = torch.zeros((6, 50)), torch.zeros((2, 3))
    p, t, o = torch.zeros((2, 4), dtype=torch.int32), torch.zeros((2, 4), dtype=torch.int32), torch.zeros((2, 4))
    ws = torch.zeros(16, dtype=torch.uint8)
    for args, kw in (((x.double(), s, p, t, o), {}), ((x[:5], s, p, t, o), {}), ((x.t().contiguous().t(), s, p, t, o), {}),
                     ((x, s.view(6), p, t, o), {}), ((x, s.double(), p, t, o), {}), ((x, s, p.long(), t, o), {}), ((x, s, p, t[:, :3], o), {}),
                     ((x, s, p, t, o.half()), {}), ((x, s, p[:1], t, o), {}), ((x, s, p, t, o), dict(done=torch.zeros(5, dtype=torch.uint8))),
                     ((x, s, p, t, o), dict(done=torch.zeros(6))), ((x, s, p, t, o), dict(dev_error=torch.zeros(1)))):
        with pytest.raises(ValueError):
            here.semkv_beam_select(*args, ws, **kw)
    with pytest.raises(here.SemkvError) as e:
        here.semkv_beam_select(x, s, p, t, o, ws)          # a workspace that is too small
    assert e.value.status == EWORKSPACE
    with pytest.raises(here.SemkvError) as e:
        here.semkv_beam_select(x[:1].expand(6, 50), s, p, t, o, ws)   # rows on one another
    assert e.value.status == EINVAL
    here.semkv_beam_select(x[:0], s[:0], p[:0], t[:0], o[:0], ws)


def test_the_binding_refuses_reorders_that_do_not_fit(here):
    c = here.KV4Cache(1, 2, 64, 16, 4, 2, 1, device="cpu")
    i32 = dict(dtype=torch.int32)
    ws = c.pages_workspace(2, 0)
    here.semkv_kv4_reorder(c, torch.zeros(0, **i32), torch.zeros(0, **i32), ws)
    for seqs, parent in ((torch.zeros(3, **i32), torch.zeros(2, **i32)), (torch.zeros(2), torch.zeros(2, **i32)), (None, torch.zeros(2))):
        with pytest.raises(ValueError):
            here.semkv_kv4_reorder(c, seqs, parent, ws)


# ------------------------------------------------- the plain forms' own pins ------

def test_the_plain_rotation_is_a_rotation():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 2, 64)).astype(np.float32)
    for pairs in (False, True):
        t = table_of(5, 32)
        y = turn(x, t, 32, pairs)
        assert np.array_equal(y[..., 32:], x[..., 32:]) and np.array_equal(y[0], x[0])
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-5)
        a, b = (0, 1) if pairs else (0, 16)
        z = (x[3, 0, a] + 1j * x[3, 0, b]) * np.exp(3j)
        assert np.allclose([y[3, 0, a], y[3, 0, b]], [z.real, z.imag], atol=1e-6)


def test_the_plain_selection_is_the_definition():
    x = torch.tensor(np.random.default_rng(1).standard_normal((6, 40)))
    s = torch.tensor([[-1.0, -2.0, -np.inf], [0.0, 0.0, -0.5]], dtype=torch.float64)
    parent, token, score = select(x.numpy(), s.numpy(), 9)
    for g in range(2):
        best, at = (torch.log_softmax(x[3 * g:3 * g + 3], 1) + s[g][:, None]).flatten().topk(9)
        assert np.allclose(score[g], best, rtol=0, atol=1e-12)
        assert np.array_equal(parent[g] * 40 + token[g], at.numpy() + 120 * g)
    parent, token, score = select(np.zeros((2, 3)), [[0.0, -1.0]], 8, done=[0, 1], end=2)
    assert parent.tolist() == [[1, 0, 0, 0, -1, -1, -1, -1]]
    assert token[0].tolist()[:4] == [2, 0, 1, 2]
