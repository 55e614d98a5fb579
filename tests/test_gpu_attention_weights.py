"""How exactly weights enter the product with the values: one-hot values show every weight by itself."""
import pytest
import torch

import kv_util as ref
from test_gpu_tree_attention import Step

pytestmark = pytest.mark.gpu


def _one_hot(fmt, counts, ctx, heads=1, group=8, dim=128, rise=0.0, seed=90):
    """At most dim positions in all; position j's value is 1 in dimension j and 0 elsewhere; scores rise by `rise` every 32."""
    s = Step(fmt, heads, group, dim, 16, [ctx], counts, trees="causal", seed=seed)
    n = ctx + counts[0]
    g = torch.Generator().manual_seed(seed)
    direction = torch.randn(1, 1, dim, generator=g)
    direction *= dim ** 0.5 / direction.norm()
    s.q[:] = (direction + 0.3 * torch.randn(s.q.shape, generator=g)).to(torch.bfloat16)
    level = rise * (torch.arange(n) // 32).float().view(-1, 1, 1)
    k = direction * dim ** -0.5 * level + 0.5 * torch.randn(n, heads, dim, generator=g)
    s.pool.write(0, torch.arange(n), k, torch.eye(n, dim)[:, None].expand(n, heads, dim))
    return s


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("rise", [0.0, 4.0, 6.5, 9.1])
@pytest.mark.parametrize("ctx,counts", [(100, [28]), (96, [5]), (120, [1])])
def test_a_weight_is_rounded_once(fmt, rise, ctx, counts):
    # `attention_bound`: the result's own rounding, one rounding of the weight, and the scores'.  A reference that moves within the
    # tile (every 32 positions here) adds none.
    s = _one_hot(fmt, counts, ctx, rise=rise, seed=90 + int(10 * rise))
    s.check()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts", [(2, 4, [1]), (1, 8, [3]), (2, 1, [20]), (2, 4, [6, 5])])
def test_few_rows_over_bf16_take_weights_of_16_bits(dim, heads, group, counts):
    # `attention_bound` with 2^-16 for a weight of two bf16 terms (2^-8 of each term, the second at most 2^-8 of the first)
    ctx = [700 + 90 * b for b in range(len(counts))]
    s = Step("bf16", heads, group, dim, 16, ctx, counts, seed=95 + dim)
    out, at = s.run().double().cpu(), 0
    for b, n in enumerate(counts):
        k, v = s.pool.rows(b, ctx[b] + n)
        want, _, mass, big = ref.attention(s.q[at:at + n], k, v, ctx[b], s.sees[b], s.scale)
        score = dim * 2.0 ** -23 * big * s.scale + 2.0 ** -20
        bound = 2.0 ** -8 * want.abs() + (2.0 ** -16 + 2 * score)[..., None] * mass
        assert bool(((out[at:at + n] - want).abs() <= bound).all())
        at += n


@pytest.mark.parametrize("dim,heads,group,counts,sms,times", [(64, 2, 4, [8], None, 1), (128, 2, 8, [3], None, 1), (64, 2, 8, [5], None, 2),
                                                              (128, 2, 8, [4], None, 2), (128, 2, 8, [40], None, 2), (64, 4, 8, [33], 1, 2)])
def test_the_error_over_bf16_on_either_side_of_the_choice_of_kernel(dim, heads, group, counts, sms, times):
    # Rounding to nearest in bf16 is off by at most 2^-8, by 2^-8 / sqrt(3) in the root of the mean square: once for the result; with
    # one-term weights once more for them, which values of random signs add up by squares as they do the result itself.  (`score`:
    # the scores' errors, as a share of sum p |v|, which exceeds the norm of the result by sqrt(n) at most.)
    from paper_2607_04031_b200 import binding as tl
    ctx = 3000
    s = Step("bf16", heads, group, dim, 16, [ctx], counts, trees="causal", seed=97 + dim)
    with tl.option(tl.OPT_SM_LIMIT, sms or 0):
        out = s.run().double().cpu()
    k, v = s.pool.rows(0, ctx + counts[0])
    want, _, mass, big = ref.attention(s.q, k, v, ctx, s.sees[0], s.scale)
    score = 2 * (dim * 2.0 ** -23 * big * s.scale + 2.0 ** -20)[..., None] * mass
    off = float((out - want).norm() / want.norm())
    assert off <= 2.0 ** -8 / 3 ** 0.5 * times ** 0.5 + float(score.norm() / want.norm())
