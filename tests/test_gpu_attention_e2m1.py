"""Attention over a 4-bit cache on the GPU, against the formula in 64 bits within the bounds of kv_util (weights as over an 8-bit cache)."""
import math

import pytest
import torch

import kv_util
import serve_util
from test_gpu_tree_attention import Step

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def four_bits(monkeypatch):
    monkeypatch.setattr(kv_util, "Pool", serve_util.Pool4)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts", [(2, 1, [1]), (1, 8, [1, 1, 1]), (4, 3, [5, 1, 2]), (2, 4, [9, 0, 16, 1]), (1, 16, [7]),
                                                (2, 8, [33, 20]), (3, 5, [64])])
def test_matches_the_formula(dim, heads, group, counts):
    ctx = [(37 * b * b + 200 * b + 3) for b in range(len(counts))]
    Step("e2m1", heads, group, dim, 32, ctx, counts, seed=dim + group).check()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts", [(2, 1, [8]), (2, 1, [9]), (1, 1, [17]), (1, 1, [24]), (2, 1, [32]), (2, 1, [33]), (1, 3, [13, 13, 13]),
                                                (1, 1, [40]), (2, 1, [47]), (1, 8, [6, 6]), (2, 1, [49]), (1, 1, [70, 1, 1]), (2, 4, [30, 1, 0, 1, 1])])
def test_rows_around_the_borders_of_blocks_and_kernels(dim, heads, group, counts):
    """Blocks of 8, 16 and 32 rows, the last one full or not, requests of fewer and of more rows than their average."""
    Step("e2m1", heads, group, dim, 32, [2900 if b == 0 else 131 * b for b in range(len(counts))], counts, trees="tree", seed=sum(counts)).check()


@pytest.mark.parametrize("ctx", [0, 1, 15, 16, 17, 63, 64, 111, 127, 128, 129, 255, 257])
@pytest.mark.parametrize("counts", [[1, 3], [40, 33]])
def test_lengths_around_every_tile_border(ctx, counts):
    Step("e2m1", 2, 4, 128, 16, [ctx, ctx + 1], counts, trees="causal", seed=ctx).check()


@pytest.mark.parametrize("counts", [[1], [8], [40]])
@pytest.mark.parametrize("page", [16, 128, 1024])
@pytest.mark.parametrize("dim", [64, 128])
def test_long_contexts_are_split_and_joined(counts, page, dim):
    Step("e2m1", 1, 4, dim, page, [9000], counts, trees="tree", seed=page).check()


@pytest.mark.parametrize("trees", ["random", "empty"])
@pytest.mark.parametrize("ctx", [0, 77])
@pytest.mark.parametrize("group,counts", [(2, [17, 3]), (8, [40, 5])])
def test_masks_of_any_bits_and_rows_that_see_nothing(trees, ctx, group, counts):
    Step("e2m1", 2, group, 128, 32, [ctx, 0], counts, trees=trees, seed=4).check()


@pytest.mark.parametrize("group,counts", [(2, [5, 9]), (8, [40, 64])])
def test_strided_pool(group, counts):
    Step("e2m1", 3, group, 128, 64, [300, 41], counts, seed=6).check(permuted=True)


@pytest.mark.parametrize("dim,group,counts", [(128, 1, [1, 4]), (64, 2, [3, 7]), (128, 8, [30, 40]), (256, 1, [2, 2])])
def test_scores_and_values_of_very_different_sizes(dim, group, counts):
    Step("e2m1", 2, group, dim, 32, [500, 700], counts, seed=8, spread=6.0).check()


@pytest.mark.parametrize("group,counts", [(1, [1]), (8, [40])])
def test_values_from_2_to_the_minus_80_to_2_to_the_100(group, counts):
    for power in (-80, -20, 60, 100):
        s = Step("e2m1", 2, group, 128, 32, [200], counts, seed=9)
        s.pool.vs = torch.where(s.pool.vs.isnan(), s.pool.vs, s.pool.vs * 2.0 ** power)
        out = s.run()
        from paper_2607_04031_b200 import binding as tl
        tl.device_status()
        if power > 60:                                       # (their bf16 results and fp64 bounds scale alike)
            assert bool(torch.isfinite(out.float()).all())
        s.compare(out.double().cpu(), s.lse.double().cpu())


@pytest.mark.parametrize("group,counts", [(2, [6]), (8, [40])])
def test_a_page_that_does_not_exist_is_not_attended_to(group, counts):
    from paper_2607_04031_b200 import binding as tl
    s = Step("e2m1", 2, group, 128, 16, [400], counts, trees="causal", seed=11)
    full = s.pool.rows(0, 400 + counts[0])
    s.pool.table[0, 3] = -5
    out = s.run()
    with pytest.raises(tl.TileLensError, match="0xa00"):
        tl.device_status()
    keep = torch.ones(400 + counts[0], dtype=torch.bool)
    keep[48:64] = False
    want, wl, mass, big = kv_util.attention(s.q, full[0][keep], full[1][keep], 400 - 16, s.sees[0], s.scale)
    bound = kv_util.attention_bound(want, mass, big, full[1], "e2m1", 128, s.scale, 400)
    assert bool(((out.double().cpu() - want).abs() <= bound).all())


@pytest.mark.parametrize("group,counts", [(2, [6, 1]), (8, [40, 9])])
def test_a_captured_step_follows_lengths_and_tables(group, counts):
    from paper_2607_04031_b200 import binding as tl
    s = Step("e2m1", 2, group, 128, 32, [900, 300], counts, trees="causal", seed=12)
    s.run()
    ws = torch.empty(max(1, tl.tree_attention_workspace_bytes(s.cache, s.batch, s.q.shape[1])), dtype=torch.uint8, device="cuda:0")
    tl.set_workspace(ws)
    try:
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=stream):
            tl.tree_attention(s.cache, s.batch, s.qd, s.out, mask=s.md, scale=s.scale, lse=s.lse)
        s.batch._tensors[1].copy_(torch.tensor([411, 17], dtype=torch.int32))
        s.out.fill_(7.0)
        graph.replay()
        tl.device_status()
    finally:
        tl.set_workspace(None)
    got = s.out.double().cpu()
    at = 0
    for b, (c, n) in enumerate(zip([411, 17], counts)):
        k, v = s.pool.rows(b, c + n)
        want, _, mass, big = kv_util.attention(s.q[at:at + n], k, v, c, s.sees[b], s.scale)
        assert bool(((got[at:at + n] - want).abs() <= kv_util.attention_bound(want, mass, big, v, "e2m1", 128, s.scale, c + n)).all())
        at += n


@pytest.mark.parametrize("group,counts", [(1, [1, 1]), (8, [30, 33])])
def test_the_same_bits_every_time(group, counts):
    s = Step("e2m1", 2, group, 128, 32, [3000, 5000], counts, seed=13)
    first = s.run().clone()
    for _ in range(3):
        assert torch.equal(s.run().view(torch.int16), first.view(torch.int16))


@pytest.mark.parametrize("group,counts", [(2, [5]), (8, [40])])
def test_a_nan_row_reaches_those_that_see_it_alone(group, counts):
    from paper_2607_04031_b200 import binding as tl
    n = counts[0]
    s = Step("e2m1", 1, group, 128, 32, [50], counts, trees="causal", seed=14)
    for scales in (s.pool.ks, s.pool.vs):
        pg, line = s.pool.place(0, torch.tensor([50 + n - 1]))
        keep = scales[pg, :, line].clone()
        scales[pg, :, line] = math.nan
        out = s.run().float().cpu()
        tl.device_status()
        assert bool(torch.isfinite(out[:n - 1]).all()) and bool(out[n - 1].isnan().all())
        scales[pg, :, line] = keep
