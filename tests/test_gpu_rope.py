"""Rotary positions on the GPU against the formula in 64 bits."""
import math

import numpy as np
import pytest
import torch

import kv_util
import serve_util as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _turns(rot, kind=0):
    from paper_2607_04031_b200 import binding as tl
    return tl.rope_turns(rot, 10000.0, kind, factor=4.0, original=2048.0, low=1.0, high=32.0 if kind == 3 else 4.0)


def _rows(dim, rot, layout, dtype, tokens, heads, positions, amplitude=1.0, inverse=False, in_place=False, pad=0, seed=0, kind=0, shift=0):
    from paper_2607_04031_b200 import binding as tl
    turns = _turns(rot, kind)
    r = tl.rope(turns.to(DEV), layout, amplitude)
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(tokens, heads, dim, generator=g).to(dtype)
    pos = torch.tensor(positions, dtype=torch.int32)
    wide = torch.full((tokens, heads * dim + pad + shift), 7.0, dtype=dtype, device=DEV)
    xd = wide[:, shift:shift + heads * dim].unflatten(1, (heads, dim))
    xd.copy_(x)
    raw = torch.full_like(wide, 7.0)
    out = xd if in_place else raw[:, shift:shift + heads * dim].unflatten(1, (heads, dim))
    tl.rope_rows(r, xd, out, pos.to(DEV), inverse=inverse)
    tl.device_status()
    want, size = ref.turned(x, turns, pos, layout, amplitude, inverse)
    bound = ref.turned_bound(want, size, amplitude, dtype)
    bound[..., rot:] = 0
    err = (out.double().cpu() - want).abs()
    assert bool((err <= bound).all()), float((err / bound.clamp_min(1e-300)).max())
    outside = (wide if in_place else raw)
    assert bool((outside[:, :shift] == 7).all()) and bool((outside[:, shift + heads * dim:] == 7).all())
    if not in_place:
        assert torch.equal(xd.cpu(), x)
    return out


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,rot", [(64, 64), (128, 128), (128, 64), (128, 32), (80, 48), (96, 16), (256, 256), (512, 512), (128, 36), (64, 2), (6, 4), (2, 2), (90, 90)])
@pytest.mark.parametrize("inverse,in_place", [(False, False), (True, True)])
def test_rows_match_the_formula(layout, dtype, dim, rot, inverse, in_place):
    pos = [0, 1, 2, 77, 5, 4095, 100000]
    _rows(dim, rot, layout, dtype, 7, 3, pos, inverse=inverse, in_place=in_place, pad=8, seed=dim + rot)


@pytest.mark.parametrize("heads", [1, 2, 5, 33, 72])
@pytest.mark.parametrize("tokens", [1, 9, 400])
def test_every_number_of_heads_and_tokens(heads, tokens):
    _rows(128, 128, 0, torch.bfloat16, tokens, heads, [(13 * i) % 4000 for i in range(tokens)])
    _rows(64, 48, 1, torch.float32, tokens, heads, [i for i in range(tokens)])


@pytest.mark.parametrize("kind", [0, 1, 2, 3])
def test_far_and_negative_positions(kind):
    _rows(128, 128, 0, torch.float32, 8, 2, [2 ** 31 - 1, -2 ** 31, -1, 2 ** 30, 10 ** 6, -77, 123456789, 3], kind=kind, amplitude=1.3)


@pytest.mark.parametrize("shift", [1, 3, 4])
def test_rows_that_no_vector_fits(shift):
    _rows(64, 64, 0, torch.bfloat16, 5, 3, [0, 1, 2, 3, 900], shift=shift, pad=3)
    _rows(64, 32, 1, torch.float32, 5, 3, [0, 1, 2, 3, 900], shift=shift, pad=5)


def test_inverse_is_the_gradient():
    """sum(g * turned(x)) has gradient turned back(g): against the formula's transpose, and against differences."""
    from paper_2607_04031_b200 import binding as tl
    for layout in (0, 1):
        turns = _turns(24)
        r = tl.rope(turns.to(DEV), layout, 1.25)
        g = torch.Generator().manual_seed(1)
        x, up = (torch.randn(4, 2, 32, generator=g) for _ in range(2))
        pos = torch.tensor([3, 0, 50, 7], dtype=torch.int32)
        grad = torch.empty(4, 2, 32, device=DEV)
        tl.rope_rows(r, up.to(DEV), grad, pos.to(DEV), inverse=True)
        step = 2.0 ** -4                                     # the map is linear: any step will do, a power of two is exact
        eye = torch.eye(32)
        f = lambda z: ref.turned(z, turns, pos, layout, 1.25)[0]  # noqa: E731
        for d in range(32):
            by = ((f(x + step * eye[d]) - f(x - step * eye[d])) / (2 * step) * up.double()).sum(-1)
            # the row's sum in fp64 against two products in fp32
            assert bool(((grad[..., d].double().cpu() - by).abs() <= 1e-5 * (1 + up.double().abs().sum(-1))).all())
        tl.device_status()


def test_rows_of_a_captured_graph_follow_positions():
    from paper_2607_04031_b200 import binding as tl
    turns = _turns(128)
    r = tl.rope(turns.to(DEV))
    x = torch.randn(6, 4, 128).to(torch.bfloat16)
    xd, pos = x.to(DEV), torch.zeros(6, dtype=torch.int32, device=DEV)
    out = torch.empty_like(xd)
    tl.rope_rows(r, xd, out, pos)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        tl.rope_rows(r, xd, out, pos)
    pos.copy_(torch.tensor([5, 1000, 3, 0, 70000, 9], dtype=torch.int32))
    graph.replay()
    tl.device_status()
    want, size = ref.turned(x, turns, pos.cpu(), 0)
    assert bool(((out.double().cpu() - want).abs() <= ref.turned_bound(want, size, 1.0, torch.bfloat16)).all())


class Append:
    def __init__(self, fmt, dim, rot, layout, dtype, heads, q_heads, page, starts, counts, seed=0):
        from paper_2607_04031_b200 import binding as tl
        g = torch.Generator().manual_seed(seed)
        total = sum(counts)
        pool = (ref.Pool4 if fmt == "e2m1" else kv_util.Pool)(fmt, heads, dim, page, [s + n for s, n in zip(starts, counts)], seed)
        self.pool, self.turns, self.starts, self.counts, self.total = pool, _turns(rot), starts, counts, total
        self.rows = torch.randn(total, q_heads + 2 * heads, dim, generator=g).to(dtype)
        self.d = self.rows.to(DEV)
        self.q, self.k, self.v = self.d[:, :q_heads], self.d[:, q_heads:q_heads + heads], self.d[:, q_heads + heads:]
        self.dev = pool.device(DEV)
        self.cache = tl.kv_cache(*self.dev)
        self.offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(DEV)
        self.batch = tl.kv_batch(pool.table.to(DEV), torch.tensor(starts, dtype=torch.int32, device=DEV), self.offsets, total)
        self.rope = tl.rope(self.turns.to(DEV), layout, 1.1)
        self.own = torch.tensor([s + i for s, n in zip(starts, counts) for i in range(n)], dtype=torch.int32)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8", "e2m1"])
@pytest.mark.parametrize("dim,rot,layout", [(64, 64, 0), (128, 128, 0), (128, 96, 1), (128, 36, 0), (256, 256, 1), (64, 30, 0), (64, 10, 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("given", [False, True])
def test_append_turns_queries_and_keys(fmt, dim, rot, layout, dtype, given):
    """Queries against the formula; what the cache holds against the formula within its own step; values as tl_kv_append leaves them."""
    from paper_2607_04031_b200 import binding as tl
    a = Append(fmt, dim, rot, layout, dtype, 3, 7, 16, [0, 5, 15, 40], [1, 0, 3, 21], seed=dim + rot)
    pos = torch.tensor([(7 * i) % 50 for i in range(a.total)], dtype=torch.int32) if given else a.own
    out = torch.full((a.total, 8, dim), 7.0, dtype=torch.bfloat16, device=DEV)
    tl.rope_append(a.cache, a.batch, a.rope, a.q, out[:, 1:], a.k, a.v, positions=pos.to(DEV) if given else None)
    back = [torch.empty(a.total, 3, dim, device=DEV) for _ in range(2)]
    tl.kv_read(a.cache, a.batch, *back)
    tl.device_status()
    rows = a.rows.double()
    want, size = ref.turned(rows[:, :7], a.turns, pos, layout, 1.1)
    assert bool(((out[:, 1:].double().cpu() - want).abs() <= ref.turned_bound(want, size, 1.1, torch.bfloat16)).all())
    assert bool((out[:, 0] == 7).all())
    want, size = ref.turned(rows[:, 7:10], a.turns, pos, layout, 1.1)
    near = ref.turned_bound(want, size, 1.1, torch.float32)
    top = want.abs().amax(-1, keepdim=True) * (1 + 2.0 ** -20)
    # half a step of the cache's rounding: relative for bf16, E4M3 (2^-4; 2^-10 of the row's largest in units of 448 where it is subnormal),
    # half of 1/127 of the largest for INT8; E2M1: half of 2 of 6 of the group's, whose scale is rounded by 2^-4 of itself, or saturates
    # by as much, and by 2^-10 of 448 where it is subnormal
    half = {"bf16": want.abs() * 2.0 ** -8, "e4m3": torch.maximum(want.abs() * 2.0 ** -4, top * 2.0 ** -10 / 448),
            "int8": top / 254, "e2m1": None}[fmt]
    if fmt == "e2m1":
        group = want.abs().unflatten(-1, (-1, 16)).amax(-1, keepdim=True).expand(*want.shape[:-1], dim // 16, 16).flatten(-2)
        half = group * (1 / 6) * (1 + 2.0 ** -4) + 6 * top * 2.0 ** -10 / 448
    assert bool(((back[0].double().cpu() - want).abs() <= half * (1 + 2.0 ** -10) + near).all())
    # values: the bits of a plain append
    b = Append(fmt, dim, rot, layout, dtype, 3, 7, 16, a.starts, a.counts, seed=dim + rot)
    tl.kv_append(b.cache, b.batch, b.k, b.v)
    for i, (x, y) in enumerate(zip(a.dev, b.dev)):
        if x is not None and i % 2 == 1:
            assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


@pytest.mark.parametrize("fmt", ["bf16", "e2m1"])
def test_append_is_turning_and_appending(fmt):
    """fp32 rows: the keys enter the cache as tl_rope_rows leaves them, bit by bit; queries turned in place, bf16."""
    from paper_2607_04031_b200 import binding as tl
    a = Append(fmt, 128, 128, 0, torch.float32, 2, 4, 32, [7, 100], [20, 3], seed=2)
    b = Append(fmt, 128, 128, 0, torch.float32, 2, 4, 32, [7, 100], [20, 3], seed=2)
    tl.rope_append(a.cache, a.batch, a.rope, None, None, a.k, a.v)
    k = torch.empty_like(b.k)
    tl.rope_rows(b.rope, b.k, k, b.own.to(DEV))
    tl.kv_append(b.cache, b.batch, k.contiguous(), b.v.contiguous())
    tl.device_status()
    for x, y in zip(a.dev, b.dev):
        if x is not None:
            assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
    for rot, layout in ((128, 0), (128, 1), (64, 0), (36, 0)):
        c = Append(fmt, 128, rot, layout, torch.bfloat16, 2, 9, 32, [7, 100], [20, 3], seed=3)
        apart = torch.empty(c.total, 9, 128, dtype=torch.bfloat16, device=DEV)
        tl.rope_append(c.cache, c.batch, c.rope, c.q, apart, c.k, c.v)
        tl.rope_append(c.cache, c.batch, c.rope, c.q, c.q, c.k, c.v)
        tl.device_status()
        assert torch.equal(apart.view(torch.int16), c.q.contiguous().view(torch.int16))


def test_append_without_a_page():
    from paper_2607_04031_b200 import binding as tl
    a = Append("e2m1", 128, 128, 0, torch.bfloat16, 2, 4, 16, [0], [40], seed=5)
    a.batch._tensors[0][0, 1] = -1
    before = [t.clone() for t in a.dev]
    out = torch.zeros(40, 4, 128, dtype=torch.bfloat16, device=DEV)
    tl.rope_append(a.cache, a.batch, a.rope, a.q, out, a.k, a.v)
    with pytest.raises(tl.TileLensError, match="0xa00"):
        tl.device_status()
    want, size = ref.turned(a.rows[:, :4].double(), a.turns, a.own, 0, 1.1)
    assert bool(((out.double().cpu() - want).abs() <= ref.turned_bound(want, size, 1.1, torch.bfloat16)).all())
    untouched = [p for p in range(a.pool.pages) if p not in a.pool.table[0, [0, 2]].tolist()]
    for t, w in zip(a.dev, before):
        assert torch.equal(t[untouched].contiguous().view(torch.uint8), w[untouched].contiguous().view(torch.uint8))


def test_positions_of_trees():
    from paper_2607_04031_b200 import binding as tl
    rng = np.random.default_rng(3)
    counts, starts = [1, 0, 17, 64, 5], [9, 4, 0, 1000, 2 ** 30]
    parents, want = [], []
    for n, s in zip(counts, starts):
        up = kv_util.random_tree(n, 3, rng) if n else []
        depth = []
        for p in up:
            depth.append(0 if p < 0 else depth[p] + 1)
        parents += up
        want += [s + d for d in depth]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    got = torch.full((sum(counts),), -7, dtype=torch.int32, device=DEV)
    tl.tree_positions(i32(parents), i32(np.concatenate([[0], np.cumsum(counts)]).tolist()), i32(starts), got)
    tl.device_status()
    assert got.tolist() == want
    # rows that no request owns are left alone
    got.fill_(-7)
    tl.tree_positions(i32(parents), i32([0, 1, 1, 3, 4, 6]), i32(starts), got)
    assert got.tolist()[6:] == [-7] * (sum(counts) - 6)
