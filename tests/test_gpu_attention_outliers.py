"""8-bit caches with one value far larger than the others, at a position that also scores high: the others still count."""
import pytest
import torch

import kv_util as ref
from test_gpu_tree_attention import Step

pytestmark = pytest.mark.gpu

# few rows; 128-row blocks; 256-row blocks (on one multiprocessor)
SHAPES = [(1, 8, [1], None), (1, 4, [3], None), (1, 8, [16], None), (2, 8, [33], 1)]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts,sms", SHAPES)
@pytest.mark.parametrize("at", ["first", "middle"])
def test_one_large_value_that_scores_high(fmt, dim, heads, group, counts, sms, at):
    # One token scores some 8 nats above the rest, and one dimension of its value is 40000 times theirs; its other dimensions are
    # zeros, so that what is in them comes from the rest alone, which hold a good part of the softmax.
    from paper_2607_04031_b200 import binding as tl
    ctx = 3000
    n = ctx + counts[0]
    s = Step(fmt, heads, group, dim, 16, [ctx], counts, trees="causal", seed=70 + dim)
    g = torch.Generator().manual_seed(71)
    direction = torch.randn(1, 1, dim, generator=g)
    direction *= dim ** 0.5 / direction.norm()
    s.q[:] = (direction + 0.05 * torch.randn(s.q.shape, generator=g)).to(torch.bfloat16)
    k = 0.3 * torch.randn(n, heads, dim, generator=g)
    v = 1.0 + 0.5 * torch.randn(n, heads, dim, generator=g)
    spot = 5 if at == "first" else ctx // 2 + 7
    k[spot] = direction[0] * 8.0 * dim ** -0.5
    v[spot] = 0
    v[spot, :, 7] = 40000.0
    s.pool.write(0, torch.arange(n), k, v)
    with tl.option(tl.OPT_SM_LIMIT, sms or 0):
        out = s.run().double().cpu()
        tl.device_status()
    pg, line = s.pool.place(0, torch.arange(n))
    kk, vv = s.pool.rows(0, n)
    codes, scales = s.pool.v.float()[pg, :, line].double().abs(), s.pool.vs[pg, :, line].double()
    want, lse, mass, big = ref.attention(s.q, kk, vv, ctx, s.sees[0], s.scale)
    assert bool((want[..., 9] > 0.2).all())                             # the rest holds a good part of the softmax
    # as `attention_bound`; a weight (taken with its value's scale, the largest being 2^7 at least) that is subnormal in f16 is off
    # by 2^-25: 2^-32 of the row's largest weight * scale for every code
    z = torch.einsum("nhd,tqhd->hqtn", kk, s.q.double().view(counts[0], heads, group, dim).permute(0, 2, 1, 3)) * s.scale
    seen = torch.ones(counts[0], n, dtype=torch.bool)
    seen[:, ctx:] = s.sees[0]
    p = torch.softmax(z.masked_fill(~seen, float("-inf")), -1)          # heads, group, tokens, positions
    largest = (p * scales.T[:, None, None]).amax(-1)
    flush = 2.0 ** -32 * torch.einsum("hqt,nhd->thqd", largest, codes).reshape(want.shape)
    score = dim * 2.0 ** -23 * big * s.scale + 2.0 ** -20
    bound = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2 * score)[..., None] * mass + flush
    err = (out - want).abs()
    assert bool((err <= bound).all()), float((err / bound).max())
