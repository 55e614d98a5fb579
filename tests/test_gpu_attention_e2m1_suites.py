"""The attention suites of the other cache formats over a 4-bit cache: prompts, blocks of 256 rows, rows apart, outliers, small values,
weights, wide tables, masks, streams, captures."""
import pytest
import torch

import kv_util
import serve_util
import test_gpu_attention_prompt as prompt
import test_gpu_attention_rows_apart as apart
import test_gpu_attention_weights as weights
import test_gpu_attention_wide_table as wide
import test_gpu_tree_attention as tree
from test_gpu_attention_e2m1_long import compare
from test_gpu_tree_attention import Step

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def four_bits(monkeypatch):
    """Pools in 4 bits, and a tighter bound: a weight is off by 2^-31 of the row's largest weight * scale at least, which scales below
    max |v| / 1344 and codes times group scales up to 2688 make 2^-30 of max |v|, each position."""
    def bound(out, mass, big, values, fmt, dim, scale, length):
        score = dim * 2.0 ** -23 * big * abs(scale) + 2.0 ** -20
        tiny = length * 2.0 ** -30 * float(values.abs().max() if values.numel() else 0.0)
        return 2.0 ** -8 * out.abs() + (2.0 ** -11 + 2 * score + length * 2.0 ** -23)[..., None] * mass + tiny + 1e-30
    monkeypatch.setattr(kv_util, "Pool", serve_util.Pool4)
    monkeypatch.setattr(kv_util, "attention_bound", bound)


@pytest.mark.parametrize("dim,heads,group,page", [(64, 1, 2, 16), (128, 1, 3, 128), (256, 1, 1, 32)])
@pytest.mark.parametrize("ctx,counts", [([0], [600]), ([800], [512]), ([0, 333, 1000], [257, 1, 130])])
def test_several_hundred_causal_rows(dim, heads, group, page, ctx, counts):
    prompt.test_several_hundred_causal_rows("e2m1", dim, heads, group, page, ctx, counts)


@pytest.mark.parametrize("dim", [64, 128])
def test_a_prompt_in_blocks_of_256_rows(dim):
    prompt.test_a_prompt_in_blocks_of_256_rows("e2m1", dim)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts,sms", apart.SHAPES + [(2, 2, [3], None), (2, 8, [4, 2], None), (2, 4, [10], None)])
@pytest.mark.parametrize("ctx", [0, 45, 400])
def test_a_token_that_a_row_does_not_see_leaves_its_bits_alone(dim, heads, group, counts, sms, ctx):
    apart.test_a_token_that_a_row_does_not_see_leaves_its_bits_alone("e2m1", dim, heads, group, counts, sms, ctx)


@pytest.mark.parametrize("rise", [0.0, 4.0, 6.5, 9.1])
@pytest.mark.parametrize("ctx,counts", [(100, [28]), (96, [5]), (120, [1])])
def test_a_weight_is_rounded_once(rise, ctx, counts):
    weights.test_a_weight_is_rounded_once("e2m1", rise, ctx, counts)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("ctx,counts,rows", [([300], [26], 128), ([300, 200], [30, 26], 128), ([4000, 2500], [30, 26], 256)])
def test_wide_tables(dim, ctx, counts, rows):
    wide.test_the_choice_of_blocks_goes_by_the_pool_where_the_table_is_wide("e2m1", dim, ctx, counts, rows)


# few rows (blocks of 8, 16, 32); 128-row blocks; 256-row blocks (on one multiprocessor)
SHAPES = [(1, 8, [1], None), (2, 4, [3], None), (1, 8, [4], None), (1, 8, [16], None), (2, 8, [33], 1)]


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts,sms", SHAPES)
@pytest.mark.parametrize("at", ["first", "middle"])
def test_one_large_value_that_scores_high(dim, heads, group, counts, sms, at):
    # one token scores some 8 nats above the rest, and one dimension of its value is 40000 times theirs
    from paper_2607_04031_b200 import binding as tl
    ctx = 3000
    n = ctx + counts[0]
    s = Step("e2m1", heads, group, dim, 16, [ctx], counts, trees="causal", seed=70 + dim)
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
        s.run()
        tl.device_status()
    compare(s)


FLOOR = 2.0 ** -98


def _small(heads, group, dim, counts, size, seed, sms):
    """Values of any size; the least scale is 2^-98, a row of zeros included."""
    from paper_2607_04031_b200 import binding as tl
    ctx = [150 + 9 * b for b in range(len(counts))]
    s = Step("e2m1", heads, group, dim, 16, ctx, counts, seed=seed)
    g = torch.Generator().manual_seed(seed)
    for b, n in enumerate(c + m for c, m in zip(ctx, counts)):
        k, _ = s.pool.rows(b, n)
        s.pool.write(b, torch.arange(n), k.float(), torch.randn(n, heads, dim, generator=g) * size(n).view(-1, 1, 1))
    with tl.option(tl.OPT_SM_LIMIT, sms or 0):
        s.run()
        tl.device_status()
    live = ~s.pool.vs.isnan()
    s.pool.vs = torch.where(live, s.pool.vs.clamp_min(FLOOR), s.pool.vs)      # (what it counts as)
    compare(s)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts,sms", SHAPES + [(2, 8, [10, 16], None)])
@pytest.mark.parametrize("size", [1e-20, 1e-24, 1e-26, 1e-28, 1e-33])
def test_values_that_are_all_small(dim, heads, group, counts, sms, size):
    _small(heads, group, dim, counts, lambda n: torch.full((n,), size), 50 + dim, sms)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts,sms", SHAPES + [(2, 8, [10, 16], None)])
def test_small_values_among_others(dim, heads, group, counts, sms):
    sizes = lambda n: torch.exp2(20.0 - 10.0 * (torch.arange(n) % 16)) * (torch.arange(n) % 7 != 3)  # noqa: E731
    _small(heads, group, dim, counts, sizes, 60 + dim, sms)


@pytest.mark.parametrize("tokens", [1, 60])
def test_the_sum_of_a_long_context_of_zeros(tokens):
    # 2^21 rows of zeros, scores just below the point where a row takes a new maximum (as for 8-bit caches; 8192 fp32 additions per
    # thread: 2^-11 of the sum)
    from paper_2607_04031_b200 import binding as tl
    page, dim, n, dev = 1024, 64, 2 ** 21, "cuda:0"
    pages = n // page + 1
    zeros = lambda *shape: torch.zeros(pages, 1, page, *shape, dtype=torch.uint8, device=dev)  # noqa: E731
    k, kg = zeros(dim // 2), zeros(dim // 16)
    k[..., 0], kg[..., 0] = 2, 0x38                          # keys: 1 in the first dimension, times their scale
    ks, vs = torch.full((pages, 1, page), 7.9 * 0.6931472, device=dev), torch.zeros(pages, 1, page, device=dev)
    ks.view(-1)[:256] = ks.view(-1)[n // 2:n // 2 + 256] = 0.0
    cache = tl.kv_cache(k, zeros(dim // 2), ks, vs, kg.view(torch.float8_e4m3fn), zeros(dim // 16).view(torch.float8_e4m3fn))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    batch = tl.kv_batch(torch.arange(pages, dtype=torch.int32, device=dev)[None], i32([n - tokens]), i32([0, tokens]), tokens)
    q = torch.zeros(tokens, 1, dim, dtype=torch.bfloat16, device=dev)
    q[..., 0] = 1
    out, lse = torch.ones_like(q), torch.zeros(tokens, 1, device=dev)
    with tl.option(tl.OPT_SM_LIMIT, 1):
        tl.tree_attention(cache, batch, q, out, scale=1.0, lse=lse)
    tl.device_status()
    z = ks.view(-1)[:n].double()
    want = torch.stack([torch.logsumexp(z[:n - tokens + i + 1], 0) for i in range(tokens)])
    assert bool((out == 0).all())
    assert bool(((lse[:, 0].double() - want).abs() <= dim * 2.0 ** -23 * 8 + 2.0 ** -20 * (1 + want.abs()) + 2.0 ** -11).all())


def test_many_units_per_cta():
    tree.test_many_units_per_cta("e2m1")


@pytest.mark.parametrize("trees", ["random", "empty", "causal"])
@pytest.mark.parametrize("ctx", [0, 50])
def test_masks(trees, ctx):
    tree.test_masks("e2m1", trees, ctx)


@pytest.mark.parametrize("counts", [[2, 1], [40, 17]])
def test_the_pool_may_be_stored_token_major(counts):
    tree.test_the_pool_may_be_stored_token_major("e2m1", counts)


@pytest.mark.parametrize("counts", [[3], [50]])
def test_large_scores(counts):
    tree.test_large_scores("e2m1", counts)


@pytest.mark.parametrize("counts", [[6], [48]])
def test_what_is_masked_has_no_influence(counts):
    tree.test_what_is_masked_has_no_influence_8_bit("e2m1", counts)


@pytest.mark.parametrize("counts", [[2], [64]])
def test_rows_of_zeros_and_mixed_scales(counts):
    tree.test_rows_of_zeros_and_mixed_scales("e2m1", counts)


@pytest.mark.parametrize("counts", [[4], [40]])
def test_a_page_outside_the_pool_is_left_out_and_reported(counts):
    tree.test_a_page_outside_the_pool_is_left_out_and_reported("e2m1", counts)


@pytest.mark.parametrize("counts", [[3, 5], [40, 64]])
def test_same_bits_every_time_and_on_another_stream(counts):
    tree.test_same_bits_every_time_and_on_another_stream(counts)


def test_a_captured_step_follows_the_lengths_on_the_device():
    tree.test_a_captured_step_follows_the_lengths_on_the_device()


def test_capture_without_a_workspace_is_refused():
    tree.test_capture_without_a_workspace_is_refused()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group,counts", [(1, 8, [16, 5, 12, 0, 16]), (2, 8, [17, 40, 33]), (1, 4, [70, 1, 64]), (1, 16, [20, 9])])
def test_many_rows_in_blocks(dim, heads, group, counts):
    tree.test_many_rows_in_blocks("e2m1", dim, heads, group, counts)


@pytest.mark.parametrize("most", [1, 12])
def test_more_requests_than_a_warp_looks_at_at_once(most):
    tree.test_more_requests_than_a_warp_looks_at_at_once("e2m1", most)


@pytest.mark.parametrize("counts", [[2], [7], [50]])
@pytest.mark.parametrize("step", [0.4, 3.0, 40.0])
def test_a_maximum_that_grows_along_the_sequence(counts, step):
    tree.test_a_maximum_that_grows_along_the_sequence("e2m1", counts, step)


@pytest.mark.parametrize("counts", [[3], [40]])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.7])
def test_any_scale(counts, scale):
    tree.test_any_scale("e2m1", counts, scale)


def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right():
    tree.test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right("e2m1")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("small,large,sms", [(4, 90, 1), (16, 60, 2), (4, 150, 1)])
def test_many_small_units_among_large_ones(dim, small, large, sms):
    tree.test_many_small_units_among_large_ones("e2m1", dim, small, large, sms)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("sms", [1, 2])
def test_units_of_one_tile_among_longer_ones(dim, sms):
    tree.test_units_of_one_tile_among_longer_ones("e2m1", dim, sms)


@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("sms", [1, 3])
def test_few_rows_on_few_multiprocessors(dim, sms):
    tree.test_few_rows_on_few_multiprocessors("e2m1", dim, sms)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("trees", ["tree", "random", "empty", "causal"])
@pytest.mark.parametrize("sms", [2, 5])
def test_blocks_of_256_rows(dim, trees, sms):
    tree.test_blocks_of_256_rows("e2m1", dim, trees, sms)


def test_pages_past_32_bit_offsets():
    from paper_2607_04031_b200 import binding as tl
    pages, page, dim, n = 36000, 1024, 256, 1500             # 4.7e9 bytes of codes, the request's pages at the end of them
    z = lambda *shape, dtype=torch.uint8: torch.empty(pages, 1, page, *shape, dtype=dtype, device="cuda")  # noqa: E731
    dev = (z(dim // 2), z(dim // 2), z(dtype=torch.float32), z(dtype=torch.float32), z(dim // 16).view(torch.float8_e4m3fn), z(dim // 16).view(torch.float8_e4m3fn))
    cache = tl.kv_cache(*dev)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    x, y = torch.randn(n, 1, dim), torch.randn(n, 1, dim)
    table = i32([[pages - 1, pages - 2]])
    tl.kv_append(cache, tl.kv_batch(table, i32([0]), i32([0, n]), n), x.cuda(), y.cuda())
    kk, vv = (serve_util.held4(*serve_util.quantise4(t)) for t in (x, y))
    scales = serve_util.quantise4(y)[2].double()
    for rows, group in ((4, 2), (1, 1), (20, 2)):
        q = torch.randn(rows, group, dim).to(torch.bfloat16)
        out = torch.empty(rows, group, dim, dtype=torch.bfloat16, device="cuda")
        tl.tree_attention(cache, tl.kv_batch(table, i32([n - rows]), i32([0, rows]), rows), q.cuda(), out)
        tl.device_status()
        sees = torch.ones(rows, rows, dtype=torch.bool).tril()
        want, _, mass, big = kv_util.attention(q, kk, vv, n - rows, sees, dim ** -0.5)
        _, largest = serve_util.weights_and_scales(q, kk, scales, n - rows, sees, dim ** -0.5)
        assert bool(((out.double().cpu() - want).abs() <= serve_util.attention_bound4(want, mass, big, largest, vv, scales, dim, dim ** -0.5)).all())
    back = [torch.empty(n, 1, dim, device="cuda") for _ in range(2)]
    tl.kv_read(cache, tl.kv_batch(table, i32([0]), i32([0, n]), n), *back)
    tl.page_copy(cache, i32([[pages - 1, 3, page], [pages - 2, pages - 3, page]]))
    tl.device_status()
    assert torch.equal(back[0].double().cpu(), kk) and torch.equal(back[1].double().cpu(), vv)
    for t in dev:
        t = t.view(torch.uint8)
        assert torch.equal(t[3], t[pages - 1]) and torch.equal(t[pages - 3], t[pages - 2])
