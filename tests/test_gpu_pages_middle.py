"""Writing in the middle of what a request holds: which rows of a replaced page its copies carry."""
import pytest
import torch

import serve_util as ref
from test_gpu_pages import Both, i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("start,tokens,pages", [(5, 10, 1), (5, 16, 1), (5, 20, 2), (16, 20, 1), (20, 33, 2), (0, 60, 4)])
def test_rows_behind_the_written_ones_of_a_replaced_page_are_not_carried(start, tokens, pages):
    # 60 positions shared by two requests; one writes start .. tokens - 1: fresh pages for those alone, the rows in front of start
    # copied into the first of them, the pages behind still shared
    from paper_2607_04031_b200 import binding as tl
    b = Both(2, 8, 40)
    b.reserve([0, -1], [60, -1])
    b.fork([0], [1], [60])
    pool = ref.Pool4("e2m1", 1, 64, 16, [40 * 16], 1, spare=0)
    dev = pool.device(DEV)
    before = [t.clone() for t in dev]
    was = b.table[0].tolist()
    tl.page_reserve(b.t, i32([-1, start]), i32([-1, tokens]), b.moves, b.n, b.m)
    moves, missing = b.plain.reserve([-1, start], [-1, tokens])
    assert missing == b.m.item() == 0
    b.same()
    first = start // 16
    now = b.table[1].tolist()
    assert [e for e in range(4) if now[e] != was[e]] == list(range(first, first + pages))
    assert moves == ([(was[first], now[first], start % 16)] if start % 16 else [])
    tl.page_copy(tl.kv_cache(*dev), b.moves, b.n)
    tl.device_status()
    for t, old in zip(dev, before):
        t, old = (z.contiguous().view(torch.uint8).view(40, 1, 16, -1) for z in (t, old))
        if start % 16:
            assert torch.equal(t[now[first], :, :start % 16], old[was[first], :, :start % 16])
            assert torch.equal(t[now[first], :, start % 16:], old[now[first], :, start % 16:])
        rest = [p for p in range(40) if p != now[first]]
        assert torch.equal(t[rest], old[rest])
