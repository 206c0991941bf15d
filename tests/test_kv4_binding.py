"""CPU checks of what the binding of the paged 4-bit cache refuses before it calls the library, and of what it
fills in.  No kernel runs: every batch here has no rows, and tensors on the CPU count as the current device's."""
import pytest
import torch


@pytest.fixture()
def sk(monkeypatch):
    from paper_2608_28911_gb300 import build
    build.build()
    from paper_2608_28911_gb300 import semkv
    monkeypatch.setattr(semkv, "_raw_device", lambda: -1)       # where CPU tensors are
    monkeypatch.setattr(semkv, "_stream", lambda stream: None)
    return semkv


class Elsewhere:
    """Stands for a tensor on another device."""
    dtype, shape = torch.int32, (2,)

    def get_device(self):
        return 1

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


def no_rows(sk):
    i32 = dict(dtype=torch.int32)
    return sk.KV4Batch(2, cu=torch.zeros(3, **i32), start=torch.zeros(2, **i32), total=0, max_count=1)


def test_a_batch_on_another_device_is_refused(sk):
    c = sk.KV4Cache(1, 2, 64, 16, 4, 2, 1, device="cpu")
    x = torch.zeros((0, 2, 64), dtype=torch.float16)
    ws = torch.zeros(64, dtype=torch.uint8)
    b = no_rows(sk)
    sk.semkv_kv4_attention(c, b, 0, x, x.clone(), 1.0, ws)
    sk.semkv_kv4_write(c, b, 0, x, x)
    b.start = Elsewhere()
    for call in (lambda: sk.semkv_kv4_attention(c, b, 0, x, x.clone(), 1.0, ws), lambda: sk.semkv_kv4_write(c, b, 0, x, x),
                 lambda: sk.semkv_kv4_read(c, b, 0, x, x.clone()), lambda: sk.semkv_kv4_reserve(c, b, ws)):
        with pytest.raises(ValueError, match="current CUDA device"):
            call()


def test_a_batch_lies_on_one_device(sk, monkeypatch):
    i32 = dict(dtype=torch.int32)
    for kw in (dict(cu=torch.zeros(3, **i32), total=0), dict(seqs=torch.zeros(2, **i32))):
        monkeypatch.setattr(sk, "_here", lambda *t: None)
        with pytest.raises(ValueError, match="one device"):
            sk.KV4Batch(2, start=Elsewhere(), **kw)


def test_buffers_that_the_library_would_refuse_make_no_cache(sk):
    """Table, length and refs carved out of one allocation: refs and pages begin on a multiple of 16 bytes."""
    store = torch.zeros(2 * 3 + 2 + 4 + 4, dtype=torch.int32)
    table, length = store[:6].view(2, 3), store[6:8]
    size = 4 * 2 * 1 * 1152
    room = torch.zeros(size + 32, dtype=torch.uint8)
    pages = room[-room.data_ptr() % 16:][:size].view(1, 4, 2, 1, 1152)
    at = -store.data_ptr() // 4 % 4 + 8             # the next multiple of 16 bytes
    c = sk.KV4Cache.over(pages, table, length, store[at:at + 4], 64)
    assert c.s.refs % 16 == 0
    for refs in (store[at - 1:at + 3], store[at - 2:at + 2]):
        with pytest.raises(ValueError, match="16 bytes"):
            sk.KV4Cache.over(pages, table, length, refs, 64)
    shifted = room[-room.data_ptr() % 16 + 4:][:size]
    with pytest.raises(ValueError, match="16 bytes"):
        sk.KV4Cache.over(shifted.view(1, 4, 2, 1, 1152), table, length, c.refs, 64)


def test_the_largest_count_of_a_step_that_names_none(sk):
    """As many rows as there are, so that no sequence is left out; one where each has one."""
    cu = torch.zeros(4, dtype=torch.int32)
    start = torch.zeros(3, dtype=torch.int32)
    assert sk.KV4Batch(3, cu=cu, start=start, total=17).s.max_count == 17
    assert sk.KV4Batch(3, cu=cu, start=start, total=17, max_count=9).s.max_count == 9
    assert sk.KV4Batch(3, cu=cu, start=start, total=0).s.max_count == 0
    assert sk.KV4Batch(3, start=start).s.max_count == 1
