"""Rows so small that their scale is a subnormal number, on the GPU: the codes are the nearest ones all the same."""
import math

import pytest
import torch

import kv_util as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_rows_whose_scale_is_subnormal(fmt, dim):
    # Largest magnitudes from one unit of 2^-149 upwards: the scale has a few bits, so that quotients reach 1.5 times the
    # largest code.  150 and 690 units are among them; the negative ones too.
    from paper_2607_04031_b200 import binding as tl
    units = torch.cat([torch.arange(1, 2049), torch.tensor([2 ** k + d for k in range(11, 24) for d in (-1, 0, 1)])])
    n = units.numel()
    g = torch.Generator().manual_seed(dim)
    rows = torch.round(units.double()[:, None, None] * (2 * torch.rand(n, 1, dim, generator=g, dtype=torch.float64) - 1))
    rows[:, 0, 5] = units.double()
    rows[:, 0, 9] = -units.double()
    rows = (rows * math.ldexp(1.0, -149)).float()
    assert float(rows[149].max()) == math.ldexp(150.0, -149)
    pool = ref.Pool(fmt, 1, dim, 64, [n], seed=1)
    batch = tl.kv_batch(pool.table.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"),
                        torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
    dev = pool.device("cuda:0")
    tl.kv_append(tl.kv_cache(*dev), batch, rows.cuda(), -rows.cuda())
    tl.device_status()
    pool.write(0, torch.arange(n), rows, -rows)
    # (the codes as bytes: an E4M3 zero's sign is part of them)
    for got, want in zip(dev, (pool.k, pool.v, pool.ks, pool.vs)):
        a, b = got.cpu().contiguous(), want.contiguous()
        if a.dtype == torch.float32:
            assert bool(((a == b) | (a.isnan() & b.isnan())).all())
        else:
            pg, line = pool.place(0, torch.arange(n))
            assert torch.equal(a.view(torch.uint8)[pg, :, line], b.view(torch.uint8)[pg, :, line])
