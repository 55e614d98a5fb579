"""Chunks of more rows than one turn of the copying kernels' grids, over several requests: every row once, and where it belongs."""
import pytest
import torch

import serve_util as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Chunk:
    """A 4-bit (or bf16) pool of zeros, requests of `counts` rows behind `starts`, pages in a random order."""

    def __init__(self, fmt, heads, dim, page, starts, counts, seed):
        from paper_2607_04031_b200 import binding as tl
        g = torch.Generator(device=DEV).manual_seed(seed)
        per = [-(-(s + n) // page) for s, n in zip(starts, counts)]
        pages, self.total, self.page = sum(per) + 3, sum(counts), page
        order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
        self.table = torch.full((len(per), max(per)), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, n in enumerate(per):
            self.table[b, :n] = order[at:at + n]
            at += n
        if fmt == "bf16":
            self.pool = [torch.zeros(pages, heads, page, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
            self.cache = tl.kv_cache(*self.pool)
        else:
            z = lambda *s, dtype=torch.uint8: torch.zeros(pages, heads, page, *s, dtype=dtype, device=DEV)  # noqa: E731
            self.pool = [z(dim // 2), z(dim // 2), z(dtype=torch.float32), z(dtype=torch.float32), z(dim // 16), z(dim // 16)]
            self.cache = tl.kv_cache(*self.pool[:4], *(t.view(torch.float8_e4m3fn) for t in self.pool[4:]))
        self.batch = tl.kv_batch(self.table, _i32(starts), _i32([sum(counts[:i]) for i in range(len(counts) + 1)]), self.total)
        self.req = torch.repeat_interleave(torch.arange(len(counts), device=DEV), torch.tensor(counts, device=DEV))
        self.pos = torch.cat([torch.arange(s, s + n, device=DEV) for s, n in zip(starts, counts)])
        self.rows = [torch.randn(self.total, heads, dim, generator=g, device=DEV) for _ in range(3)]

    def at(self):
        return self.table[self.req, self.pos // self.page].long(), self.pos % self.page


CASES = [(16, 64, 32, [5, 0, 700], [20001, 1, 19998]), (8, 256, 16, [0, 33], [12000, 8007]), (3, 128, 64, [100, 7, 0, 50], [30000, 0, 33, 25001])]


@pytest.mark.parametrize("heads,dim,page,starts,counts", CASES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_and_read(heads, dim, page, starts, counts, dtype):
    from paper_2607_04031_b200 import binding as tl
    c = Chunk("e2m1", heads, dim, page, starts, counts, seed=dim)
    k, v = (t.to(dtype) for t in c.rows[:2])
    tl.kv_append(c.cache, c.batch, k, v)
    back = [torch.full((c.total, heads, dim), 7.0, dtype=dtype, device=DEV) for _ in range(2)]
    tl.kv_read(c.cache, c.batch, *back)
    tl.device_status()
    want = [torch.zeros_like(t) for t in c.pool]
    pg, line = c.at()
    for i, x in enumerate((k, v)):
        codes, group, scale = ref.quantise4(x)
        for t, w in ((want[i], codes), (want[2 + i], scale), (want[4 + i], group)):
            t[pg, :, line] = w
        held = ref.held4(codes.cpu()[::97], group.cpu()[::97], scale.cpu()[::97])
        assert torch.equal(back[i][::97].double().cpu(), held)
    for got, w in zip(c.pool, want):
        assert torch.equal(got, w)


@pytest.mark.parametrize("fmt", ["bf16", "e2m1"])
@pytest.mark.parametrize("heads,dim,page,starts,counts", CASES)
@pytest.mark.parametrize("layout", [0, 1])
def test_turned_and_appended(fmt, heads, dim, page, starts, counts, layout):
    """The keys of tl_rope_append as tl_rope_rows leaves them and tl_kv_append takes them, bit by bit; queries likewise."""
    from paper_2607_04031_b200 import binding as tl
    one, two = (Chunk(fmt, heads, dim, page, starts, counts, seed=dim + 1) for _ in range(2))
    rope = tl.rope(tl.rope_turns(dim).to(DEV), layout)
    q, k, v = one.rows
    out = torch.full((one.total, heads, dim), 7.0, dtype=torch.bfloat16, device=DEV)
    tl.rope_append(one.cache, one.batch, rope, q, out, k, v)
    turned = [torch.empty_like(t) for t in (q, k)]
    for x, y in zip((q, k), turned):
        tl.rope_rows(rope, x, y, one.pos.to(torch.int32))
    tl.kv_append(two.cache, two.batch, turned[1], v)
    tl.device_status()
    assert torch.equal(out, turned[0].to(torch.bfloat16))
    for a, b in zip(one.pool, two.pool):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
