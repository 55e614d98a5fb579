"""8-bit caches with very small values and rows of zeros: what the smallest scale does to results and sums."""
import pytest
import torch

import kv_util as ref
from test_gpu_tree_attention import Step

pytestmark = pytest.mark.gpu

# few rows; 128-row blocks; 256-row blocks (on one multiprocessor)
SHAPES = [(2, 4, [3], None), (1, 8, [4], None), (2, 8, [10, 16], None), (4, 4, [60], 1)]
FLOOR = 2.0 ** -90


def _step(fmt, heads, group, dim, counts, size, seed, ctx=150):
    ctx = [ctx + 9 * b for b in range(len(counts))]
    s = Step(fmt, heads, group, dim, 16, ctx, counts, seed=seed)
    g = torch.Generator().manual_seed(seed)
    for b, n in enumerate(c + m for c, m in zip(ctx, counts)):
        k, _ = s.pool.rows(b, n)
        s.pool.write(b, torch.arange(n), k.float(), torch.randn(n, heads, dim, generator=g) * size(n).view(-1, 1, 1))
    return s


def _check(s, fmt, sms):
    """Against fp64 with scales of 2^-90 at least.  As `attention_bound`; a weight that is subnormal in f16 is off by 2^-25, a code
    counts at most the largest scale and the sum at least 1 of it."""
    from paper_2607_04031_b200 import binding as tl
    with tl.option(tl.OPT_SM_LIMIT, sms or 0):
        out = s.run().double().cpu()
        tl.device_status()
    lse, at = s.lse.double().cpu(), 0
    for b, n in enumerate(s.counts):
        length = s.ctx[b] + n
        pg, line = s.pool.place(b, torch.arange(length))
        k, _ = s.pool.rows(b, length)
        scales = s.pool.vs[pg, :, line].double().clamp_min(FLOOR)
        v = s.pool.v.float()[pg, :, line].double() * scales[..., None]
        want, wl, mass, big = ref.attention(s.q[at:at + n], k, v, s.ctx[b], s.sees[b], s.scale)
        step = 2.0 ** -25 * float(scales.max()) * ref.TOP[fmt] * length
        score = s.dim * 2.0 ** -23 * big * s.scale + 2.0 ** -20
        bound = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2 * score)[..., None] * mass + step
        err = (out[at:at + n] - want).abs()
        assert bool((err <= bound).all()), float((err / bound).max())
        room = s.dim * 2.0 ** -23 * big * s.scale + 2.0 ** -20 * (1 + wl.abs())
        assert bool(((lse[at:at + n] - wl).abs() <= room).all())
        at += n


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts,sms", SHAPES)
@pytest.mark.parametrize("size", [1e-20, 1e-24, 1e-26, 5e-29, 1e-36])
def test_values_that_are_all_small(fmt, dim, heads, group, counts, sms, size):
    _check(_step(fmt, heads, group, dim, counts, lambda n: torch.full((n,), size), seed=50 + dim), fmt, sms)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts,sms", SHAPES)
def test_small_values_among_others(fmt, dim, heads, group, counts, sms):
    # neighbours of every size from 2^-130 to 2^20, and rows of zeros
    sizes = lambda n: torch.exp2(20.0 - 10.0 * (torch.arange(n) % 16)) * (torch.arange(n) % 7 != 3)  # noqa: E731
    _check(_step(fmt, heads, group, dim, counts, sizes, seed=60 + dim), fmt, sms)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("tokens", [1, 48])
def test_the_sum_of_a_long_context_of_zeros(fmt, tokens):
    # 2^21 rows of zeros.  Where a CTA begins the scores are 0, from there on just below the point where a row takes a new maximum:
    # every weight is as large as it gets, and so is its share of the sum.  (8192 fp32 additions per thread: 2^-11 of the sum.)
    from paper_2607_04031_b200 import binding as tl
    page, heads, dim, n = 1024, 1, 64, 2 ** 21
    dev = "cuda:0"
    code = torch.float8_e4m3fn if fmt == "e4m3" else torch.int8
    pool = torch.zeros(n // page + 1, heads, page, dim, device=dev).to(code)
    one = torch.ones(1, device=dev).to(code)
    pool.view(torch.uint8)[..., 0] = one.view(torch.uint8)                  # keys: 1 in the first dimension, times their scale
    ks = torch.full(pool.shape[:3], 7.9 * 0.6931472, device=dev)            # scores of 7.9 in log2
    vs = torch.zeros(pool.shape[:3], device=dev)
    table = torch.arange(n // page + 1, dtype=torch.int32, device=dev)[None]
    ks.view(-1)[:256] = ks.view(-1)[n // 2:n // 2 + 256] = 0.0
    offs = torch.tensor([0, tokens], dtype=torch.int32, device=dev)
    batch = tl.kv_batch(table, torch.tensor([n - tokens], dtype=torch.int32, device=dev), offs, tokens)
    zeros = torch.zeros(pool.shape, device=dev).to(code)
    cache = tl.kv_cache(pool, zeros, ks, vs)
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
