"""The paged 4-bit cache on the GPU where its format and its softmax have their ends."""
import numpy as np
import pytest

from kv4_plain import Plain
from test_gpu_kv4 import cu_of, make

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
