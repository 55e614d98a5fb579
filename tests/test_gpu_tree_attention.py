"""Tree attention over the paged cache on the GPU, against a plain fp64 statement within bounds derived in kv_util."""
import math

import numpy as np
import pytest
import torch

import kv_util as ref

pytestmark = pytest.mark.gpu

FORMATS = ["bf16", "e4m3", "int8"]


class Step:
    """One step: a filled pool, queries, masks; runs the library and checks every row."""

    def __init__(self, fmt, heads, group, dim, page, ctx, counts, trees="tree", seed=0, words=None, spread=1.0):
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.fmt, self.heads, self.group, self.dim, self.ctx, self.counts = fmt, heads, group, dim, list(ctx), list(counts)
        self.pool = ref.Pool(fmt, heads, dim, page, [c + n for c, n in zip(ctx, counts)], seed)
        for b, n in enumerate(c + n for c, n in zip(ctx, counts)):
            if n:
                k = torch.randn(n, heads, dim, generator=g) * spread
                v = torch.randn(n, heads, dim, generator=g) * torch.exp(torch.randn(n, heads, 1, generator=g))
                self.pool.write(b, torch.arange(n), k, v)
        total = sum(counts)
        self.q = torch.randn(total, heads * group, dim, generator=g).to(torch.bfloat16)
        most = max(counts)
        self.words = words or max(1, -(-most // 32))
        self.sees = []
        rows = []
        for n in counts:
            if trees == "tree":
                bits = ref.tree_bits(ref.random_tree(n, 3, rng) if n else [], self.words)
            elif trees == "random":
                bits = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (n, self.words)).astype(np.int32))
            elif trees == "empty":
                bits = torch.zeros(n, self.words, dtype=torch.int32)
            else:
                bits = None
            if bits is None:
                self.sees.append(torch.ones(n, n, dtype=torch.bool).tril())
            else:
                rows.append(bits)
                j = torch.arange(n)
                inside = j < 32 * self.words
                w = bits.long()[:, (j // 32).clamp_max(self.words - 1)] >> (j % 32)
                self.sees.append(((w & 1) == 1) & inside)
        self.mask = torch.cat(rows) if rows else None
        self.scale = dim ** -0.5

    def run(self, permuted=False, stream=None, workspace=None, lse=True, q=None):
        from paper_2607_04031_b200 import binding as tl
        dev = "cuda:0"
        total, hq = self.q.shape[:2]
        self.dev = self.pool.device(dev, permuted)
        self.cache = tl.kv_cache(*self.dev)
        offs = torch.tensor(np.concatenate([[0], np.cumsum(self.counts)]).astype(np.int32)).to(dev)
        self.batch = tl.kv_batch(self.pool.table.to(dev), torch.tensor(self.ctx, dtype=torch.int32, device=dev), offs, total)
        # queries and results as column ranges of wider rows
        wide = torch.full((total, (hq + 1) * self.dim), 7.0, dtype=torch.bfloat16, device=dev)
        qd = wide[:, self.dim:].view(total, hq, self.dim)
        qd.copy_(self.q.to(dev))
        self.raw = torch.full((total + 2, hq * self.dim + 8), 7.0, dtype=torch.bfloat16, device=dev)
        out = self.raw[1:-1, 8:].view(total, hq, self.dim)
        self.lse = torch.full((total, hq), 7.0, device=dev) if lse else None
        self.qd, self.md = qd, None if self.mask is None else self.mask.to(dev)
        tl.tree_attention(self.cache, self.batch, qd, out, mask=self.md, scale=self.scale, lse=self.lse)
        self.out = out
        return out

    def check(self, **kw):
        from paper_2607_04031_b200 import binding as tl
        out = self.run(**kw)
        tl.device_status()
        assert bool((self.raw[0] == 7).all()) and bool((self.raw[-1] == 7).all()) and bool((self.raw[:, :8] == 7).all())
        self.compare(out.double().cpu(), self.lse.double().cpu())

    def compare(self, out, lse):
        at = 0
        for b, n in enumerate(self.counts):
            if n == 0:
                continue
            k, v = self.pool.rows(b, self.ctx[b] + n)
            want, wl, mass, big = ref.attention(self.q[at:at + n], k, v, self.ctx[b], self.sees[b], self.scale)
            bound = ref.attention_bound(want, mass, big, v, self.fmt, self.dim, self.scale, self.ctx[b] + n)
            err = (out[at:at + n] - want).abs()
            assert bool((err <= bound).all()), (b, float((err / bound).max()))
            seen = wl > -math.inf
            assert torch.equal(lse[at:at + n] > -math.inf, seen)
            assert bool((out[at:at + n][~seen] == 0).all())
            off = (lse[at:at + n] - wl)[seen].abs()
            room = (self.dim * 2.0 ** -23 * big * self.scale + 2.0 ** -20 * (1 + wl.abs()))[seen]
            assert bool((off <= room).all())
            at += n


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts", [(2, 1, [1]), (1, 8, [1, 1, 1]), (4, 3, [5, 1, 2]), (2, 4, [9, 0, 16, 1]), (1, 16, [7]),
                                                (2, 8, [33, 20]), (3, 5, [64])])
def test_matches_the_formula(fmt, dim, heads, group, counts):
    ctx = [(37 * b * b + 200 * b + 3) for b in range(len(counts))]
    Step(fmt, heads, group, dim, 32, ctx, counts, seed=dim + group).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("ctx", [0, 1, 15, 16, 17, 63, 64, 111, 112, 127, 128, 129, 255, 257])
def test_lengths_around_every_tile_border(fmt, ctx):
    Step(fmt, 2, 4, 128, 16, [ctx, ctx + 1], [1, 3], trees="causal", seed=ctx).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts", [[1], [8], [40]])
@pytest.mark.parametrize("page", [16, 128, 1024])
def test_long_contexts_are_split_and_joined(fmt, counts, page):
    Step(fmt, 1, 4, 128, page, [9000], counts, trees="tree", seed=page).check()


@pytest.mark.parametrize("fmt", FORMATS)
def test_many_units_per_cta(fmt):
    counts = [1 + (7 * b) % 5 for b in range(150)]
    Step(fmt, 4, 2, 64, 16, [(53 * b) % 300 for b in range(150)], counts, seed=5).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("trees", ["random", "empty", "causal"])
@pytest.mark.parametrize("ctx", [0, 50])
def test_masks(fmt, trees, ctx):
    # random bits (rows that do not see themselves), bits past the words, rows that see nothing at all
    Step(fmt, 2, 3, 128, 16, [ctx, 0, 0], [70, 33, 1], trees=trees, seed=11).check()
    if trees == "random":
        Step(fmt, 2, 3, 128, 16, [ctx, 0], [70, 40], trees=trees, seed=12, words=1).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts", [[2, 1], [40, 17]])
def test_the_pool_may_be_stored_token_major(fmt, counts):
    Step(fmt, 4, 2, 128, 32, [100, 77], counts, seed=3).check(permuted=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts", [[3], [50]])
def test_large_scores(fmt, counts):
    # scores of several hundred: a softmax that is nearly one-hot, with a maximum that keeps growing along the sequence
    s = Step(fmt, 2, 4, 128, 16, [700], counts, seed=13, spread=40.0)
    s.check()


@pytest.mark.parametrize("counts", [[6], [48]])
def test_what_is_masked_has_no_influence_bf16(counts):
    # token 2's key and value hold infinities and NaN; rows that do not see it are as without it
    n = counts[0]
    clean = Step("bf16", 2, 4, 128, 16, [45], counts, seed=21)
    dirty = Step("bf16", 2, 4, 128, 16, [45], counts, seed=21)
    pg, line = dirty.pool.place(0, torch.tensor([45 + 2]))
    dirty.pool.v[pg, :, line] = math.inf
    dirty.pool.v[pg, 0, line, 7] = math.nan
    dirty.pool.k[pg, 1, line] = math.nan
    a, b = clean.run().float().cpu(), dirty.run().float().cpu()
    hidden = ~clean.sees[0][:, 2]
    assert bool(hidden.any()) and bool((~hidden).any())
    # (weights may stay unrounded on the path that keeps such values out: 2^-8 of sum p |v| <= max |v|, and each result's
    # own rounding, 2^-8 of it in one and in the other)
    top = float(clean.pool.rows(0, 45 + n)[1].abs().max())
    assert bool(((a - b)[hidden].abs() <= 2.0 ** -7 * a[hidden].abs() + 2.0 ** -8 * top).all())
    seen = b[~hidden]
    assert bool((~torch.isfinite(seen)).all())
    assert bool(seen[:, :4, 7].isnan().all()) and bool((seen[:, :4, :7] == math.inf).all()) and bool(seen[:, 4:].isnan().all())


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("counts", [[6], [48]])
def test_what_is_masked_has_no_influence_8_bit(fmt, counts):
    clean = Step(fmt, 2, 4, 128, 16, [45], counts, seed=21)
    dirty = Step(fmt, 2, 4, 128, 16, [45], counts, seed=21)
    pg, line = dirty.pool.place(0, torch.tensor([45 + 2]))
    bad = torch.full((1, 2, 128), math.nan)
    dirty.pool.write(0, torch.tensor([45 + 2]), bad, bad)              # scale NaN, codes 0
    a, b = clean.run().float().cpu(), dirty.run().float().cpu()
    hidden = ~clean.sees[0][:, 2]
    assert torch.equal(a[hidden], b[hidden])
    assert bool(b[~hidden].isnan().all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts", [[2], [64]])
def test_rows_of_zeros_and_mixed_scales(fmt, counts):
    s = Step(fmt, 1, 8, 128, 16, [150], counts, seed=31)
    z = torch.zeros(1, 1, 128)
    for pos in (0, 5, 149):
        s.pool.write(0, torch.tensor([pos]), torch.randn(1, 1, 128), z)            # a value of zeros keeps its weight
        s.pool.write(0, torch.tensor([pos + 1]), z, torch.randn(1, 1, 128) * 1e4)  # a large value behind a zero key
    s.q[0, 0] = 0                                                                   # a query of zeros: the plain mean
    s.check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts", [[4], [40]])
def test_a_page_outside_the_pool_is_left_out_and_reported(fmt, counts):
    from paper_2607_04031_b200 import binding as tl
    s = Step(fmt, 2, 2, 128, 16, [100], counts, trees="causal", seed=2)
    s.pool.table[0, 2] = s.pool.pages + 5
    out = s.run().double().cpu()
    with pytest.raises(tl.TileLensError, match="a00"):
        tl.device_status()
    s.pool.table[0, 2] = 0
    k, v = s.pool.rows(0, 100 + counts[0])
    keep = torch.ones(100 + counts[0], dtype=torch.bool)
    keep[32:48] = False
    want, wl, mass, big = ref.attention(s.q, k[keep], v[keep], 84, s.sees[0], s.scale)
    assert bool(((out - want).abs() <= ref.attention_bound(want, mass, big, v[keep], fmt, 128, s.scale, 100)).all())


@pytest.mark.parametrize("counts", [[3, 5], [40, 64]])
def test_same_bits_every_time_and_on_another_stream(counts):
    s = Step("e4m3", 4, 4, 128, 32, [3000, 1200], counts, seed=9)
    a = s.run().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = s.run().clone()
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, s.run())


def test_a_captured_step_follows_the_lengths_on_the_device():
    from paper_2607_04031_b200 import binding as tl
    s = Step("int8", 2, 4, 128, 32, [2000, 900], [5, 5], trees="causal", seed=6)
    s.check()
    need = tl.tree_attention_workspace_bytes(s.cache, s.batch, s.q.shape[1])
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    start = s.batch._tensors[1]
    graph = torch.cuda.CUDAGraph()
    tl.set_workspace(ws)
    try:
        with torch.cuda.graph(graph):
            tl.tree_attention(s.cache, s.batch, s.qd, s.out, scale=s.scale, lse=s.lse)
    finally:
        tl.set_workspace(None)
    for ctx in ([2000, 900], [17, 850], [0, 0]):
        start.copy_(torch.tensor(ctx, dtype=torch.int32))
        s.out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        s.ctx = ctx
        s.compare(s.out.double().cpu(), s.lse.double().cpu())
    tl.device_status()


def test_capture_without_a_workspace_is_refused():
    from paper_2607_04031_b200 import binding as tl
    s = Step("int8", 2, 4, 128, 32, [2000], [5], trees="causal", seed=6)
    s.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.out.fill_(1.0)
        with pytest.raises(tl.TileLensError) as e:
            tl.tree_attention(s.cache, s.batch, s.qd, s.out, scale=s.scale)
    assert e.value.status == 6


def test_pages_past_32_bit_offsets():
    from paper_2607_04031_b200 import binding as tl
    pages, page, dim = 20000, 1024, 256
    k = torch.empty(pages, 1, page, dim, dtype=torch.int8, device="cuda")
    v = torch.empty_like(k)
    ks, vs = (torch.empty(pages, 1, page, device="cuda") for _ in range(2))
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    n = 1500
    offs = lambda m: torch.tensor([0, m], dtype=torch.int32, device="cuda")  # noqa: E731
    x, y = torch.randn(n, 1, dim), torch.randn(n, 1, dim)
    cache = tl.kv_cache(k, v, ks, vs)
    tl.kv_append(cache, tl.kv_batch(table, torch.zeros(1, dtype=torch.int32, device="cuda"), offs(n), n), x.cuda(), y.cuda())
    q = torch.randn(4, 2, dim).to(torch.bfloat16)
    out = torch.empty(4, 2, dim, dtype=torch.bfloat16, device="cuda")
    tl.tree_attention(cache, tl.kv_batch(table, torch.tensor([n - 4], dtype=torch.int32, device="cuda"), offs(4), 4), q.cuda(), out)
    tl.device_status()
    kk, vv = (ref.held(*ref.quantise(t, "int8")) for t in (x, y))
    want, _, mass, big = ref.attention(q, kk, vv, n - 4, torch.ones(4, 4, dtype=torch.bool).tril(), dim ** -0.5)
    assert bool(((out.double().cpu() - want).abs() <= ref.attention_bound(want, mass, big, vv, "int8", dim, dim ** -0.5, n)).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group,counts", [(1, 8, [16, 5, 12, 0, 16]), (2, 8, [17, 40, 33]), (1, 4, [70, 1, 64]), (1, 16, [20, 9])])
def test_many_rows_in_blocks(fmt, dim, heads, group, counts):
    # 40 to 640 rows a request: one block of 128, one of 256 of which half or a few rows are used, several blocks
    ctx = [130 * b + 61 for b in range(len(counts))]
    Step(fmt, heads, group, dim, 16, ctx, counts, seed=dim + group + len(counts)).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("most", [1, 12])
def test_more_requests_than_a_warp_looks_at_at_once(fmt, most):
    counts = [(5 * b) % (most + 1) for b in range(75)]
    Step(fmt, 2, 4, 64, 16, [(31 * b) % 200 for b in range(75)], counts, trees="causal", seed=8).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts", [[2], [50]])
@pytest.mark.parametrize("step", [0.4, 3.0, 40.0])
def test_a_maximum_that_grows_along_the_sequence(fmt, counts, step):
    # every 16 positions the scores rise by a little, or by much, so that the running maximum is taken anew within tiles
    # and between them
    s = Step(fmt, 1, 4, 128, 16, [620], counts, seed=17)
    g = torch.Generator().manual_seed(5)
    direction = torch.randn(1, 1, 128, generator=g)
    s.q[:] = (direction * 128 ** 0.5 / direction.norm() + 0.1 * torch.randn(s.q.shape, generator=g)).to(torch.bfloat16)
    n = 620 + counts[0]
    pos = torch.arange(n)
    k = direction * (step * (pos // 16).float()).view(-1, 1, 1) / direction.norm() + 0.1 * torch.randn(n, 1, 128, generator=g)
    s.pool.write(0, pos, k, torch.randn(n, 1, 128, generator=g))
    s.check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts", [[3], [40]])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.7])
def test_any_scale(fmt, counts, scale):
    from paper_2607_04031_b200 import binding as tl
    s = Step(fmt, 2, 4, 128, 32, [300], counts, seed=23)
    s.scale = scale
    out = s.run()
    tl.device_status()
    if scale < 0:
        # (q . k) * scale = (-q . k) * -scale: the bounds of the comparison are stated for scales that are not negative
        s.q, s.scale = -s.q, -scale
    s.compare(out.double().cpu(), s.lse.double().cpu())


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(fmt):
    from paper_2607_04031_b200 import binding as tl
    s = Step(fmt, 2, 4, 128, 16, [500], [40], seed=3)
    s.check()
    with tl.option(tl.OPT_WAIT_LIMIT_US, 20000):
        tl.set_option(tl.OPT_STALL_ONCE, 5)
        s.run()
        with pytest.raises(tl.TileLensError, match="c00"):
            tl.device_status()
    assert tl.get_option(tl.OPT_STALL_ONCE) == 0
    s.check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("small,large", [(4, 90), (16, 60), (4, 150), (16, 110)])
@pytest.mark.parametrize("sms", [1, 2])
def test_many_small_units_among_large_ones(fmt, dim, small, large, sms):
    # blocks of 256 rows by the average; most units have at most 128, several in a row in every CTA
    from paper_2607_04031_b200 import binding as tl
    counts = [small if b % 6 else large for b in range(1, 13)]
    with tl.option(tl.OPT_SM_LIMIT, sms):
        Step(fmt, 2, 8, dim, 16, [(29 * b) % 110 for b in range(12)], counts, trees="causal", seed=small + dim).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("sms", [1, 2])
def test_units_of_one_tile_among_longer_ones(fmt, dim, sms):
    # blocks of 128 rows; the second stream has no tile in most units, several in a row in every CTA
    from paper_2607_04031_b200 import binding as tl
    with tl.option(tl.OPT_SM_LIMIT, sms):
        Step(fmt, 2, 8, dim, 16, [(29 * b) % 110 if b % 5 else 300 for b in range(15)], [5 + b % 3 for b in range(15)], seed=dim).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("sms", [1, 3])
def test_few_rows_on_few_multiprocessors(fmt, dim, sms):
    from paper_2607_04031_b200 import binding as tl
    with tl.option(tl.OPT_SM_LIMIT, sms):
        Step(fmt, 2, 4, dim, 16, [(61 * b) % 230 for b in range(20)], [1 + b % 3 for b in range(20)], seed=dim).check()


def block_rows(s, sms):
    """Query rows of a unit, from the workspace that calls on `sms` multiprocessors ask for (tcgen05: one CTA each)."""
    from paper_2607_04031_b200 import binding as tl
    row = 2 * sms * (s.dim * 4 + 8)
    need = tl.tree_attention_workspace_bytes(s.cache, s.batch, s.q.shape[1])
    assert need % row == 0
    return need // row


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("trees", ["tree", "random", "empty", "causal"])
@pytest.mark.parametrize("sms", [2, 5])
def test_blocks_of_256_rows(fmt, dim, trees, sms):
    # 320 and 208 rows: a block and a quarter, and one not quite full
    from paper_2607_04031_b200 import binding as tl
    s = Step(fmt, 4, 8, dim, 16, [700, 333], [40, 26], trees=trees, seed=dim + sms)
    with tl.option(tl.OPT_SM_LIMIT, sms):
        s.check()
        assert block_rows(s, sms) == 256


@pytest.mark.parametrize("fmt", FORMATS)
def test_blocks_of_256_rows_and_what_is_masked(fmt):
    # token 2's key and value hold what is not finite; rows that do not see it are as without it
    from paper_2607_04031_b200 import binding as tl
    clean, dirty = (Step(fmt, 4, 4, 128, 16, [400], [60], seed=22) for _ in range(2))
    bad = torch.full((1, 4, 128), math.nan)
    if fmt == "bf16":
        pg, line = dirty.pool.place(0, torch.tensor([402]))
        dirty.pool.v[pg, :, line] = math.inf
        dirty.pool.k[pg, 1, line] = math.nan
    else:
        dirty.pool.write(0, torch.tensor([402]), bad, bad)
    with tl.option(tl.OPT_SM_LIMIT, 1):
        a, b = clean.run().float().cpu(), dirty.run().float().cpu()
    hidden = ~clean.sees[0][:, 2]
    assert bool(hidden.any()) and bool((~hidden).any())
    # (bf16: weights may stay unrounded on the path that keeps such values out)
    room = 2.0 ** -7 * a.abs() + 2.0 ** -8 * float(clean.pool.rows(0, 460)[1].abs().max()) if fmt == "bf16" else torch.zeros_like(a)
    assert bool(((a - b).abs() <= room)[hidden].all())
    assert bool((~torch.isfinite(b[~hidden])).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts,sms,rows", [([24, 24], 2, 256), ([23, 23], 2, 128), ([24, 24], 100, 128)])
def test_the_choice_of_blocks_does_not_show(fmt, counts, sms, rows):
    from paper_2607_04031_b200 import binding as tl
    s = Step(fmt, 4, 8, 128, 16, [300, 290], counts, seed=5)
    with tl.option(tl.OPT_SM_LIMIT, sms):
        s.check()
        if sms == 2:
            assert block_rows(s, sms) == rows


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tokens", [2, 3, 4, 5])
def test_rows_around_the_choice_of_kernel(fmt, dim, tokens):
    # 16 to 40 rows per key/value head, in a batch whose requests have fewer and more than the average
    Step(fmt, 2, 8, dim, 32, [700, 65, 0], [tokens - 1, tokens, tokens + 1], seed=tokens).check()


def test_a_batch_of_too_many_tiles_is_refused():
    # 2^16 requests whose tables have room for 2^26 positions each: no memory is looked at
    from paper_2607_04031_b200 import binding as tl
    s = Step("int8", 2, 4, 128, 1024, [100], [1], seed=1)
    s.check()
    b = tl.KvBatch()
    b.page_table, b.start, b.token_offsets = s.batch.page_table, s.batch.start, s.batch.token_offsets
    b.table_stride, b.requests, b.tokens = 2 ** 16, 2 ** 16, 2 ** 16
    b._ref = tl.ctypes.byref(b)
    assert tl.tree_attention_workspace_bytes(s.cache, b, 8) == 0
    q = torch.empty(2 ** 16, 8, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(tl.TileLensError) as e:
        tl.tree_attention(s.cache, b, q, torch.empty_like(q))
    assert e.value.status == 2


@pytest.mark.parametrize("counts", [[3], [50]])
def test_the_workspace_may_be_the_callers(counts):
    from paper_2607_04031_b200 import binding as tl
    s = Step("e4m3", 2, 4, 128, 32, [3000], counts, seed=12)
    a = s.run().clone()
    need = tl.tree_attention_workspace_bytes(s.cache, s.batch, s.q.shape[1])
    ws = torch.full((need + 256,), 7, dtype=torch.uint8, device="cuda")
    try:
        tl.set_workspace(ws[:need])
        assert torch.equal(a, s.run())
        assert bool((ws[need:] == 7).all()) and not bool((ws[:need] == 7).all())
        tl.set_workspace(ws[:need - 256])
        with pytest.raises(tl.TileLensError) as e:
            s.run()
        assert e.value.status == 6
    finally:
        tl.set_workspace(None)
