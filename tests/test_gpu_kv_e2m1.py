"""The 4-bit key/value cache on the GPU: writes, reads, commits and page copies against the rule, bit by bit."""
import math

import numpy as np
import pytest
import torch

import serve_util as ref

pytestmark = pytest.mark.gpu


def _bytes(t):
    return t.contiguous().view({1: torch.uint8, 4: torch.int32}[t.element_size()]).cpu()


def _same(got, want):
    """Equal bits, any NaN for a NaN."""
    if got.dtype is torch.float32:
        a, b = got.cpu(), want
        return bool(((a == b) | (a.isnan() & b.isnan())).all())
    return torch.equal(_bytes(got), _bytes(want))


def _step(pool, starts, counts, rows, dev="cuda:0"):
    """rows [tokens, 2, heads, dim] as column ranges of one product's output."""
    from paper_2607_04031_b200 import binding as tl
    total, wide = sum(counts), pool.heads * pool.dim
    out = torch.full((total, 2 * wide + 16), 9.0, dtype=rows.dtype, device=dev)
    out[:, 16:] = rows.to(dev).reshape(total, 2 * wide)
    k, v = out[:, 16:16 + wide].view(total, pool.heads, pool.dim), out[:, 16 + wide:].view(total, pool.heads, pool.dim)
    offs = torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(dev)
    return k, v, tl.kv_batch(pool.table.to(dev), torch.tensor(starts, dtype=torch.int32, device=dev), offs, total)


def _all(pool):
    return pool.k, pool.v, pool.ks, pool.vs, pool.kg, pool.vg


@pytest.mark.parametrize("dim,heads,page,permuted", [(64, 3, 16, False), (128, 8, 32, False), (256, 1, 64, False), (128, 2, 1024, True), (64, 5, 32, True)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_writes_the_rule_and_nothing_else_and_reads_it_back(dim, heads, page, permuted, dtype):
    from paper_2607_04031_b200 import binding as tl
    starts, counts = [0, 5, page - 1, 40, 3 * page], [1, 0, 3, 37, 2]
    pool = ref.Pool4("e2m1", heads, dim, page, [s + n for s, n in zip(starts, counts)], seed=dim + page)
    g = torch.Generator().manual_seed(7)
    # rows of very different sizes, and channels within them
    rows = torch.randn(sum(counts), 2, heads, dim, generator=g) * torch.exp(4 * torch.randn(sum(counts), 2, heads, 1, generator=g)) * \
        torch.exp(torch.randn(dim, generator=g))
    rows = rows.to(dtype)
    k, v, batch = _step(pool, starts, counts, rows)
    dev = pool.device("cuda:0", permuted)
    cache = tl.kv_cache(*dev)
    tl.kv_append(cache, batch, k, v)
    back = [torch.full((sum(counts), heads, dim), 7.0, dtype=dtype, device="cuda:0") for _ in range(2)]
    tl.kv_read(cache, batch, *back)
    tl.device_status()
    at = 0
    for b, (s, n) in enumerate(zip(starts, counts)):
        pool.write(b, torch.arange(s, s + n), rows[at:at + n, 0], rows[at:at + n, 1])
        if n:
            want = [side[s:] for side in pool.rows(b, s + n)]
            assert all(torch.equal(t[at:at + n].double().cpu(), w) for t, w in zip(back, want))       # (exact in bf16 too)
        at += n
    for got, want in zip(dev, _all(pool)):
        assert _same(got, want)


def test_append_special_rows():
    from paper_2607_04031_b200 import binding as tl
    dim, page = 128, 16
    rows = torch.zeros(14, 1, dim)
    rows[1] = 1e-42                                   # subnormal: everything underflows
    rows[2] = torch.linspace(-3, 3, dim)
    rows[3, 0, 5] = math.inf
    rows[4, 0, 5] = -math.inf
    rows[5, 0, 127] = math.nan
    rows[6] = 3.4e38
    rows[7] = torch.arange(dim).float() / 16          # many quotients halfway between two codes
    rows[8, 0, 64] = -1e-30
    rows[9, 0, :16], rows[9, 0, 16:] = 1.0, 2.0 ** -18      # groups whose scale is near E4M3's last step, and below it
    rows[10, 0, :16], rows[10, 0, 16:] = 1.0, 2.0 ** -22
    rows[11] = 2688.0                                 # exactly 6 * 448: scale 1; and the next number above
    rows[12] = torch.nextafter(torch.tensor(2688.0), torch.tensor(3000.0))
    rows[13] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 16) * 13.0
    pool = ref.Pool4("e2m1", 1, dim, page, [14], seed=1)
    both = torch.stack([rows, rows.flip(0)], 1)
    k, v, batch = _step(pool, [0], [14], both)
    dev = pool.device("cuda:0")
    cache = tl.kv_cache(*dev)
    tl.kv_append(cache, batch, k, v)
    back = [torch.full((14, 1, dim), 7.0, device="cuda:0") for _ in range(2)]
    tl.kv_read(cache, batch, *back)
    tl.device_status()
    pool.write(0, torch.arange(14), both[:, 0], both[:, 1])
    for got, want in zip(dev, _all(pool)):
        assert _same(got, want)
    got, (want, _) = back[0].double().cpu(), pool.rows(0, 14)
    for i in range(14):
        if i in (3, 4, 5):
            assert bool(got[i].isnan().all())
        else:
            assert torch.equal(got[i], want[i].float().double())
    # half a step at most of what the row's codes can hold there
    for i in (2, 7, 11, 13):
        assert bool(((got[i] - rows[i].double()).abs() <= rows[i].double().abs().unflatten(-1, (-1, 16)).amax(-1, keepdim=True).expand(-1, -1, 16).flatten(-2) * (1 / 6 + 1 / 16)).all())


def test_read_takes_any_group_byte_for_a_finite_scale():
    from paper_2607_04031_b200 import binding as tl
    pool = ref.Pool4("e2m1", 2, 64, 16, [64], seed=3)
    pool.ks.fill_(0.5), pool.vs.fill_(2.0)
    pool.kg.view(-1)[:256] = torch.arange(256, dtype=torch.uint8)[torch.randperm(256)]
    dev = pool.device("cuda:0")
    cache = tl.kv_cache(*dev)
    batch = tl.kv_batch(pool.table.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda:0"), torch.tensor([0, 64], dtype=torch.int32, device="cuda:0"), 64)
    back = [torch.zeros(64, 2, 64, device="cuda:0") for _ in range(2)]
    tl.kv_read(cache, batch, *back)
    tl.device_status()
    for t, w in zip(back, pool.rows(0, 64)):
        assert torch.equal(t.double().cpu(), w)


@pytest.mark.parametrize("dim,heads,page", [(64, 3, 16), (128, 8, 32), (256, 2, 64)])
def test_commit_moves_codes_and_both_scales(dim, heads, page):
    from paper_2607_04031_b200 import binding as tl
    starts, counts = [3, page - 2, 40], [9, 17, 1]
    accepted = [[0, 2, 5, 8], [0, 1, 15, 16, 16], [0]]
    accepted[1] = [0, 3, 4, 16]
    pool = ref.Pool4("e2m1", heads, dim, page, [s + n for s, n in zip(starts, counts)], seed=dim)
    dev = pool.device("cuda:0")
    cache = tl.kv_cache(*dev)
    offs = torch.tensor([0, 9, 26, 27], dtype=torch.int32, device="cuda:0")
    batch = tl.kv_batch(pool.table.cuda(), torch.tensor(starts, dtype=torch.int32, device="cuda:0"), offs, 27)
    acc = torch.full((3, 5), -1, dtype=torch.int32)
    for b, a in enumerate(accepted):
        acc[b, :len(a)] = torch.tensor(a, dtype=torch.int32)
    new = torch.zeros(3, dtype=torch.int32, device="cuda:0")
    tl.kv_commit(cache, batch, acc.cuda(), torch.tensor([len(a) for a in accepted], dtype=torch.int32, device="cuda:0"), new)
    tl.device_status()
    for b, a in enumerate(accepted):
        src = [starts[b] + i for i in a]
        pg, line = pool.place(b, torch.tensor(src))
        pt, to = pool.place(b, starts[b] + torch.arange(len(a)))
        for t in _all(pool):
            t[pt, :, to] = t[pg, :, line].clone()
    for got, want in zip(dev, _all(pool)):
        assert _same(got, want)
    assert new.tolist() == [s + len(a) for s, a in zip(starts, accepted)]


def test_positions_without_a_page_are_left_out_and_reported():
    from paper_2607_04031_b200 import binding as tl
    pool = ref.Pool4("e2m1", 2, 128, 16, [40], seed=5)
    pool.table[0, 1] = pool.pages
    rows = torch.randn(40, 2, 2, 128)
    k, v, batch = _step(pool, [0], [40], rows)
    dev = pool.device("cuda:0")
    cache = tl.kv_cache(*dev)
    tl.kv_append(cache, batch, k, v)
    with pytest.raises(tl.TileLensError, match="0xa00"):
        tl.device_status()
    back = [torch.full((40, 2, 128), 7.0, device="cuda:0") for _ in range(2)]
    tl.kv_read(cache, batch, *back)
    with pytest.raises(tl.TileLensError, match="0xa00"):
        tl.device_status()
    pos = torch.cat([torch.arange(16), torch.arange(32, 40)])
    pool.write(0, pos, rows[pos, 0], rows[pos, 1])
    for got, want in zip(dev, _all(pool)):
        assert _same(got, want)
    assert bool((back[0][16:32] == 0).all())
