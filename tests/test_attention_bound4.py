"""The bound that attention over a 4-bit cache is held to at long contexts is broken by any 16 positions that go missing."""
import math

import pytest
import torch

import kv_util
import serve_util as ref


def marked_values(n, heads, dim, g):
    """Values that say where they come from: 16 positions share a dimension of their own among dim neighbours of theirs."""
    at = (torch.arange(n) // 16) % dim
    v = torch.zeros(n, heads, dim)
    size = (1.0 + torch.rand(n, heads, generator=g)) * torch.where(torch.rand(n, heads, generator=g) < 0.5, -1.0, 1.0)
    v[torch.arange(n), :, at] = size
    # (all of one sign within the 16, so that they do not cancel)
    sign = torch.where(torch.rand(-(-n // 16), heads, generator=g) < 0.5, -1.0, 1.0)
    return v.abs() * sign.repeat_interleave(16, 0)[:n, :, None]


@pytest.mark.parametrize("dim,n", [(64, 3000), (128, 9000)])
def test_sixteen_positions_that_go_missing_break_the_bound(dim, n):
    g = torch.Generator().manual_seed(3)
    pool = ref.Pool4("e2m1", 1, dim, 16, [n], seed=2)
    pool.write(0, torch.arange(n), torch.randn(n, 1, dim, generator=g), marked_values(n, 1, dim, g))
    k, v = pool.rows(0, n)
    pg, line = pool.place(0, torch.arange(n))
    scales = pool.vs[pg, :, line].double()
    q = torch.randn(1, 2, dim, generator=g).to(torch.bfloat16)
    sees = torch.ones(1, 1, dtype=torch.bool)
    want, _, mass, big = kv_util.attention(q, k, v, n - 1, sees, dim ** -0.5)
    p, largest = ref.weights_and_scales(q, k, scales, n - 1, sees, dim ** -0.5)
    bound = ref.attention_bound4(want, mass, big, largest, v, scales, dim, dim ** -0.5)
    for first in range(0, n, 16):
        part = torch.einsum("qj,jd->qd", p[:, 0, first:first + 16], v[first:first + 16, 0])
        assert bool((part.abs() > 4 * bound[0]).any(-1).all()), first
    # and the same 16 read twice, or another 16's values in their place
    for first, other in ((0, 16), (16 * 40, 16 * 41), (0, n // 32 * 16)):
        part = torch.einsum("qj,jd->qd", p[:, 0, first:first + 16], v[other:other + 16, 0] - v[first:first + 16, 0])
        assert bool((part.abs() > 4 * bound[0]).any(-1).all())


def test_largest_product_and_shares():
    q = torch.tensor([[[1.0, 0.0]]]).to(torch.bfloat16)
    k = torch.tensor([[[0.0, 5.0]], [[math.log(3.0), 0.0]], [[9.0, 9.0]]], dtype=torch.float64)
    p, largest = ref.weights_and_scales(q, k, torch.tensor([[8.0], [2.0], [1e9]], dtype=torch.float64), 2, torch.zeros(1, 1, dtype=torch.bool), 1.0)
    assert torch.allclose(p, torch.tensor([[[0.25, 0.75, 0.0]]], dtype=torch.float64)) and abs(float(largest) - 2.0) < 1e-12
