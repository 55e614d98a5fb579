"""The paged key/value cache on the GPU: quantised writes, reads, commits and tree masks against plain statements."""
import math

import numpy as np
import pytest
import torch

import kv_util as ref

pytestmark = pytest.mark.gpu

FORMATS = ["bf16", "e4m3", "int8"]


def _step(pool, starts, counts, seed, dtype=torch.bfloat16, dev="cuda:0"):
    """A step's K and V as column ranges of one product's output."""
    from paper_2607_04031_b200 import binding as tl
    g = torch.Generator().manual_seed(seed)
    total, wide = sum(counts), pool.heads * pool.dim
    out = (torch.randn(total, 2 * wide + 16, generator=g) * 3).to(dtype)
    k, v = out[:, 16:16 + wide].view(total, pool.heads, pool.dim), out[:, 16 + wide:].view(total, pool.heads, pool.dim)
    d = out.to(dev)
    kd, vd = d[:, 16:16 + wide].view(total, pool.heads, pool.dim), d[:, 16 + wide:].view(total, pool.heads, pool.dim)
    offs = torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(dev)
    batch = tl.kv_batch(pool.table.to(dev), torch.tensor(starts, dtype=torch.int32, device=dev), offs, total)
    return k, v, kd, vd, batch


def _bits(t):
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()]).cpu()


def _same(got, want):
    """Equal bits, any NaN for a NaN."""
    if got.dtype.is_floating_point:
        a, b = got.float().cpu(), want.float()
        return bool(((a == b) | (a.isnan() & b.isnan())).all())
    return torch.equal(got.cpu(), want)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim,heads,page", [(64, 3, 16), (128, 8, 32), (256, 1, 64), (128, 2, 1024)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_writes_the_rule_and_nothing_else(fmt, dim, heads, page, dtype):
    from paper_2607_04031_b200 import binding as tl
    starts, counts = [0, 5, page - 1, 40, 3 * page], [1, 0, 3, 37, 2]
    pool = ref.Pool(fmt, heads, dim, page, [s + n for s, n in zip(starts, counts)], seed=dim + page)
    k, v, kd, vd, batch = _step(pool, starts, counts, seed=7, dtype=dtype)
    dev = pool.device("cuda:0")
    tl.kv_append(tl.kv_cache(*dev), batch, kd, vd)
    tl.device_status()
    at = 0
    for b, (s, n) in enumerate(zip(starts, counts)):
        pool.write(b, torch.arange(s, s + n), k[at:at + n], v[at:at + n])
        at += n
    for got, want in zip(dev, (pool.k, pool.v, pool.ks, pool.vs)):
        assert got is None or _same(got, want)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_special_rows(fmt):
    from paper_2607_04031_b200 import binding as tl
    dim, page = 128, 16
    rows = torch.zeros(9, 1, dim)
    rows[1] = 1e-42                                   # subnormal: the scale underflows
    rows[2] = torch.linspace(-3, 3, dim)
    rows[3, 0, 5] = math.inf
    rows[4, 0, 5] = -math.inf
    rows[5, 0, 127] = math.nan
    rows[6] = 3e38
    rows[7] = torch.arange(dim).float() / 127 * 0.5   # many quotients halfway between two codes
    rows[8, 0, 64] = -1e-30
    pool = ref.Pool(fmt, 1, dim, page, [9], seed=1)
    batch = tl.kv_batch(pool.table.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"),
                        torch.tensor([0, 9], dtype=torch.int32, device="cuda"), 9)
    dev = pool.device("cuda:0")
    cache = tl.kv_cache(*dev)
    tl.kv_append(cache, batch, rows.cuda(), rows.flip(0).cuda())
    back = [torch.full((9, 1, dim), 7.0, device="cuda") for _ in range(2)]
    tl.kv_read(cache, batch, *back)
    tl.device_status()
    pool.write(0, torch.arange(9), rows, rows.flip(0))
    for got, want in zip(dev, (pool.k, pool.v, pool.ks, pool.vs)):
        assert _same(got, want)
    for x, got in ((rows, back[0].cpu()), (rows.flip(0), back[1].cpu())):
        for i in range(9):
            if not bool(torch.isfinite(x[i]).all()):
                assert bool(got[i].isnan().all())
                continue
            s = float(x[i].abs().max()) / ref.TOP[fmt]
            # half a step of the code: INT8 0.5, E4M3 2^-4 of the value or half its smallest subnormal, 2^-10; a row too
            # small for its scale reads back as zeros
            step = 0.5 * s if fmt == "int8" else (x[i].abs() * 2.0 ** -4).clamp_min(2.0 ** -10 * s)
            assert bool(((got[i] - x[i]).abs() <= step * (1 + 2.0 ** -18) + 2e-38 * 2.0 ** -12).all()), i


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("permuted", [False, True])
def test_read_gives_what_the_codes_stand_for(fmt, out, permuted):
    from paper_2607_04031_b200 import binding as tl
    lengths = [1, 0, 100, 33, 64]
    pool = ref.Pool(fmt, 4, 128, 32, lengths, seed=3)
    g = torch.Generator().manual_seed(4)
    for b, n in enumerate(lengths):
        pool.write(b, torch.arange(n), torch.randn(n, 4, 128, generator=g), torch.randn(n, 4, 128, generator=g) * 0.1)
    total = sum(lengths)
    offs = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()
    batch = tl.kv_batch(pool.table.cuda(), torch.zeros(5, dtype=torch.int32, device="cuda"), offs, total)
    wide = torch.full((total + 2, 2, 4 * 128), 7.0, dtype=out, device="cuda")
    k, v = wide[1:-1, 0].view(total, 4, 128), wide[1:-1, 1].view(total, 4, 128)
    tl.kv_read(tl.kv_cache(*pool.device("cuda:0", permuted)), batch, k, v)
    tl.device_status()
    want = [torch.cat([pool.rows(b, n)[i] for b, n in enumerate(lengths)]).float().to(out) for i in range(2)]
    assert _same(k, want[0]) and _same(v, want[1])
    assert bool((wide[0] == 7).all()) and bool((wide[-1] == 7).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim,heads,page", [(64, 2, 16), (128, 8, 32), (256, 3, 16)])
def test_commit_moves_the_kept_rows(fmt, dim, heads, page):
    from paper_2607_04031_b200 import binding as tl
    rng = np.random.default_rng(dim)
    starts, counts = [0, 9, page - 2, 100, 7, 15], [20, 1, 12, 0, 64, 33]
    pool = ref.Pool(fmt, heads, dim, page, [s + n for s, n in zip(starts, counts)], seed=5)
    g = torch.Generator().manual_seed(6)
    for b, (s, n) in enumerate(zip(starts, counts)):
        pool.write(b, torch.arange(s + n), torch.randn(s + n, heads, dim, generator=g), torch.randn(s + n, heads, dim, generator=g))
    # chains of sources that are destinations of later entries, everything kept, one kept, nothing
    keep = [[0, 3, 4, 5, 9, 10, 19], [0], list(range(12)), [], sorted([0] + rng.choice(np.arange(1, 64), 40, replace=False).tolist()),
            [0, 32]]
    accepted = torch.full((6, 64), -1, dtype=torch.int32)
    for b, a in enumerate(keep):
        accepted[b, :len(a)] = torch.tensor(a, dtype=torch.int32)
    n_acc = torch.tensor([len(a) for a in keep], dtype=torch.int32)
    dev = pool.device("cuda:0")
    start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    offs = torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
    batch = tl.kv_batch(pool.table.cuda(), start, offs, sum(counts))
    tl.kv_commit(tl.kv_cache(*dev), batch, accepted.cuda(), n_acc.cuda(), start)         # the new lengths over the old ones
    tl.device_status()
    assert start.cpu().tolist() == [s + len(a) for s, a in zip(starts, keep)]
    for t in (pool.k, pool.v, pool.ks, pool.vs):
        if t is None:
            continue
        t = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
        for b, a in enumerate(keep):
            src_pg, src_line = pool.place(b, starts[b] + torch.tensor(a, dtype=torch.long))
            moved = t[src_pg, :, src_line].clone()
            dst_pg, dst_line = pool.place(b, starts[b] + torch.arange(len(a)))
            t[dst_pg, :, dst_line] = moved
    for got, want in zip(dev, (pool.k, pool.v, pool.ks, pool.vs)):
        assert got is None or _same(got, want)


def test_commit_skips_and_reports_what_it_cannot_move():
    from paper_2607_04031_b200 import binding as tl
    pool = ref.Pool("int8", 1, 64, 16, [16], seed=8)
    pool.write(0, torch.arange(8), torch.randn(8, 1, 64), torch.randn(8, 1, 64))
    dev = pool.device("cuda:0")
    batch = tl.kv_batch(pool.table.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"),
                        torch.tensor([0, 8], dtype=torch.int32, device="cuda"), 8)
    acc = torch.tensor([[0, 9, 1, 5]], dtype=torch.int32, device="cuda")                 # 9: no such row; 1 < 2
    tl.kv_commit(tl.kv_cache(*dev), batch, acc, torch.tensor([4], dtype=torch.int32, device="cuda"))
    with pytest.raises(tl.TileLensError, match="b00"):
        tl.device_status()
    pg = int(pool.table[0, 0])
    want = pool.k[pg].clone()
    want[:, 3] = want[:, 5]
    assert torch.equal(dev[0][pg].cpu(), want)
    tl.device_status()                                                                   # the report was taken


@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_bad_pages_are_not_touched_and_reported(bad):
    from paper_2607_04031_b200 import binding as tl
    pool = ref.Pool("e4m3", 2, 128, 16, [48], seed=9)
    pool.table[0, 1] = bad
    k, v, kd, vd, batch = _step(pool, [0], [48], seed=2)
    dev = pool.device("cuda:0")
    cache = tl.kv_cache(*dev)
    tl.kv_append(cache, batch, kd, vd)
    with pytest.raises(tl.TileLensError, match="a00"):
        tl.device_status()
    back = [torch.full((48, 2, 128), 7.0, device="cuda") for _ in range(2)]
    tl.kv_read(cache, batch, *back)
    with pytest.raises(tl.TileLensError, match="a00"):
        tl.device_status()
    assert bool((back[0][16:32] == 0).all()) and not bool((back[0][:16] == 0).all()) and not bool((back[1][32:] == 0).all())


def test_positions_past_the_table_are_refused_on_the_device():
    from paper_2607_04031_b200 import binding as tl
    pool = ref.Pool("bf16", 1, 64, 16, [32], seed=9)
    k, v, kd, vd, batch = _step(pool, [30], [4], seed=2)
    dev = pool.device("cuda:0")
    tl.kv_append(tl.kv_cache(*dev), batch, kd, vd)
    with pytest.raises(tl.TileLensError, match="a00"):
        tl.device_status()
    pool.write(0, torch.arange(30, 32), k[:2], v[:2])
    assert _same(dev[0], pool.k) and _same(dev[1], pool.v)


def test_pages_past_32_bit_offsets():
    from paper_2607_04031_b200 import binding as tl
    pages, page, dim = 20000, 1024, 256                                                   # 5.2 GB of keys, as much of values
    k = torch.empty(pages, 1, page, dim, dtype=torch.int8, device="cuda")
    v = torch.empty_like(k)
    ks, vs = (torch.empty(pages, 1, page, device="cuda") for _ in range(2))
    table = torch.tensor([[pages - 1, 17, pages - 2]], dtype=torch.int32, device="cuda")
    n = 3 * page
    batch = tl.kv_batch(table, torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
    x, y = torch.randn(n, 1, dim, device="cuda"), torch.randn(n, 1, dim, device="cuda")
    cache = tl.kv_cache(k, v, ks, vs)
    tl.kv_append(cache, batch, x, y)
    back = [torch.empty_like(x), torch.empty_like(y)]
    tl.kv_read(cache, batch, *back)
    tl.device_status()
    for a, got in ((x, back[0]), (y, back[1])):
        c, s = ref.quantise(a.cpu(), "int8")
        assert torch.equal(got.cpu(), ref.held(c, s).float())
    assert bool((v[pages - 1, 0, 5].cpu() == ref.quantise(y[5].cpu(), "int8")[0]).all())


@pytest.mark.parametrize("counts,words", [([1], 1), ([5, 0, 33, 64, 1], 2), ([100, 7], 3), ([70], 4)])
def test_tree_mask(counts, words):
    from paper_2607_04031_b200 import binding as tl
    rng = np.random.default_rng(sum(counts))
    trees = [ref.random_tree(n, 3, rng) if n else [] for n in counts]
    parents = torch.tensor([p for t in trees for p in t], dtype=torch.int32, device="cuda")
    offs = torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
    mask = torch.full((sum(counts), words), -7, dtype=torch.int32, device="cuda")
    tl.tree_mask(parents, offs, mask)
    want = torch.cat([ref.tree_bits(t, words) for t in trees if t])
    assert torch.equal(mask.cpu(), want)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_codes_are_those_of_the_exact_quotient(fmt):
    # A million quotients, bf16 (whose ratios often lie on, or next to, the middle between two codes) and fp32, at scales
    # from the smallest normal numbers to the largest: every code is the division's.
    from paper_2607_04031_b200 import binding as tl
    for dtype in (torch.bfloat16, torch.float32):
        g = torch.Generator().manual_seed(12)
        x = torch.randn(4096, 1, 256, generator=g) * torch.exp2(torch.randint(-120, 120, (4096, 1, 1), generator=g).float())
        x = x.to(dtype)
        pool = ref.Pool(fmt, 1, 256, 64, [4096], seed=1)
        batch = tl.kv_batch(pool.table.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"),
                            torch.tensor([0, 4096], dtype=torch.int32, device="cuda"), 4096)
        dev = pool.device("cuda:0")
        tl.kv_append(tl.kv_cache(*dev), batch, x.cuda(), x.cuda())
        tl.device_status()
        pool.write(0, torch.arange(4096), x, x)
        for got, want in zip(dev, (pool.k, pool.v, pool.ks, pool.vs)):
            assert _same(got, want)
