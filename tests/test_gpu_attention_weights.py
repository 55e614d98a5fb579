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
