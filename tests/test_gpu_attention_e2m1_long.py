"""Attention over a 4-bit cache at long contexts, within the bound that 16 missing positions break (test_attention_bound4)."""
import pytest
import torch

import kv_util
import serve_util
from test_attention_bound4 import marked_values
from test_gpu_tree_attention import Step, block_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def four_bits(monkeypatch):
    monkeypatch.setattr(kv_util, "Pool", serve_util.Pool4)


def compare(s):
    """Results and lse of a step that has run."""
    out, lse, at = s.out.double().cpu(), s.lse.double().cpu(), 0
    for b, n in enumerate(s.counts):
        if n == 0:
            continue
        length = s.ctx[b] + n
        k, v = s.pool.rows(b, length)
        pg, line = s.pool.place(b, torch.arange(length))
        scales = s.pool.vs[pg, :, line].double()
        q = s.q[at:at + n]
        want, wl, mass, big = kv_util.attention(q, k, v, s.ctx[b], s.sees[b], s.scale)
        _, largest = serve_util.weights_and_scales(q, k, scales, s.ctx[b], s.sees[b], s.scale)
        bound = serve_util.attention_bound4(want, mass, big, largest, v, scales, s.dim, s.scale)
        err = (out[at:at + n] - want).abs()
        assert bool((err <= bound).all()), (b, float((err / bound).max()))
        seen = wl > -float("inf")
        assert torch.equal(lse[at:at + n] > -float("inf"), seen) and bool((out[at:at + n][~seen] == 0).all())
        room = (s.dim * 2.0 ** -23 * big * s.scale + 2.0 ** -20 * (1 + wl.abs()) + length * 2.0 ** -23)[seen]
        assert bool(((lse[at:at + n] - wl)[seen].abs() <= room).all())
        at += n


def step(heads, group, dim, page, ctx, counts, marked, seed, trees="tree"):
    s = Step("e2m1", heads, group, dim, page, ctx, counts, trees=trees, seed=seed)
    if marked:
        g = torch.Generator().manual_seed(seed)
        for b, n in enumerate(c + m for c, m in zip(ctx, counts)):
            s.pool.write(b, torch.arange(n), torch.randn(n, heads, dim, generator=g), marked_values(n, heads, dim, g))
    return s


# blocks of 8, 16 and 32 rows, tcgen05 with 128 rows
@pytest.mark.parametrize("group,counts", [(4, [1]), (4, [4]), (4, [8]), (2, [26])])
@pytest.mark.parametrize("page", [16, 1024])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("marked", [False, True])
def test_long_contexts(group, counts, page, dim, marked):
    from paper_2607_04031_b200 import binding as tl
    s = step(1, group, dim, page, [9000], counts, marked, seed=page + dim)
    s.run()
    tl.device_status()
    compare(s)


@pytest.mark.parametrize("sms", [1, 3])
@pytest.mark.parametrize("group,counts", [(4, [1, 2]), (4, [7, 3]), (8, [6, 2])])
@pytest.mark.parametrize("marked", [False, True])
def test_many_tiles_for_every_cta(sms, group, counts, marked):
    from paper_2607_04031_b200 import binding as tl
    s = step(2, group, 128, 32, [5000, 3333], counts, marked, seed=sms)
    with tl.option(tl.OPT_SM_LIMIT, sms):
        s.run()
        tl.device_status()
    compare(s)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("marked", [False, True])
def test_long_contexts_in_blocks_of_256_rows(dim, marked):
    from paper_2607_04031_b200 import binding as tl
    sms = 2
    s = step(1, 8, dim, 64, [2300, 1111], [30, 26], marked, seed=dim)
    with tl.option(tl.OPT_SM_LIMIT, sms):
        s.run()
        tl.device_status()
        assert block_rows(s, sms) == 256
    compare(s)
