"""Zeros with a sign in the 4-bit cache: the code keeps the sign of x / (group scale * scale), as the plain rule does."""
import math

import pytest
import torch

import serve_util as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rows(dim, dtype):
    """Rows with zeros of either sign, values that vanish beside the largest, and a row of nothing but -0."""
    x = torch.randn(6, 2, 2, dim, generator=torch.Generator().manual_seed(dim))
    x[0, ..., ::3] = -0.0
    x[1, ..., 1::4], x[1, ..., 2::4] = 0.0, -0.0
    x[2] = -0.0
    x[3, ..., :16] = -0.0                                    # a group scale of 0 beside others
    x[4, ..., 0], x[4, ..., 1::2] = 2.0 ** 120, -1e-30        # -1e-30 * 2^-109 is below fp32's least number: it rounds to -0
    x[5, ..., 5] = -0.0
    x[5, ..., 17] = -math.inf
    return x.to(dtype)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("call", ["append", "rope_append"])
def test_a_zero_keeps_its_sign(dim, dtype, call):
    from paper_2607_04031_b200 import binding as tl
    pool = ref.Pool4("e2m1", 2, dim, 16, [6], seed=1)
    rows = _rows(dim, dtype)
    dev = pool.device(DEV)
    cache = tl.kv_cache(*dev)
    batch = tl.kv_batch(pool.table.to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV), torch.tensor([0, 6], dtype=torch.int32, device=DEV), 6)
    k, v = (rows[:, i].contiguous().to(DEV) for i in range(2))
    if call == "append":
        tl.kv_append(cache, batch, k, v)
    else:                                                    # (its values are not turned)
        tl.rope_append(cache, batch, tl.rope(tl.rope_turns(dim).to(DEV)), None, None, k, v)
    tl.device_status()
    pool.write(0, torch.arange(6), rows[:, 0], rows[:, 1])
    assert bool((pool.v[pool.table[0, 0].long()] & 15 == 8).any())
    sides = ((dev[1], pool.v), (dev[5].view(torch.uint8), pool.vg)) + (((dev[0], pool.k), (dev[4].view(torch.uint8), pool.kg)) if call == "append" else ())
    for got, want in sides:
        assert torch.equal(got.cpu(), want)
