"""What the page calls and the 4-bit cache refuse before any CUDA call."""
import ctypes

import pytest

P, Q = 0x10000, 0x900000


@pytest.fixture(scope="module")
def tl():
    from paper_2607_04031_b200 import build
    build.build()
    from paper_2607_04031_b200 import binding
    return binding


def _tables(tl, **kw):
    t = tl.PageTables()
    for name, value in {**dict(page_table=P, held=P, holders=P, table_stride=8, requests=3, pages=100, page_tokens=32), **kw}.items():
        setattr(t, name, value)
    return ctypes.byref(t)


@pytest.mark.parametrize("change,status", [(dict(page_table=None), 1), (dict(held=None), 1), (dict(holders=None), 1), (dict(table_stride=0), 1),
                                           (dict(requests=-1), 1), (dict(pages=0), 1), (dict(page_tokens=0), 1), (dict(page_tokens=8), 2),
                                           (dict(page_tokens=48), 2), (dict(page_tokens=2048), 2), (dict(pages=2 ** 30 + 1), 2),
                                           (dict(table_stride=2 ** 30 + 1), 2), (dict(page_table=P + 2), 3), (dict(held=P + 1), 3),
                                           (dict(holders=P + 2), 3)])
def test_tables_that_are_refused(tl, change, status):
    L = tl.lib()
    assert L.tl_page_reserve(_tables(tl, **change), P, P, P, P, P, None) == status
    assert L.tl_page_release(_tables(tl, **change), P, None) == status
    assert L.tl_page_fork(_tables(tl, **change), P, P, P, 2, None) == status
    assert L.tl_page_compact(_tables(tl, **change), P, 4, P, P, None) == status
    assert L.tl_page_workspace_bytes(_tables(tl, **change), 0) == 0


def test_arguments(tl):
    L, t = tl.lib(), _tables(tl)
    for i in range(5):
        a = [None if k == i else P for k in range(5)]
        assert L.tl_page_reserve(t, *a, None) == 1
        a = [P + 2 if k == i else P for k in range(5)]
        assert L.tl_page_reserve(t, *a, None) == 3
    assert L.tl_page_release(t, P + 2, None) == 3 and L.tl_page_release(_tables(tl, requests=0), None, None) == 0
    assert L.tl_page_fork(t, None, P, P, 1, None) == 1 and L.tl_page_fork(t, P, None, P, 1, None) == 1 and L.tl_page_fork(t, P, P, None, 1, None) == 1
    assert L.tl_page_fork(t, P, P, P, -1, None) == 1 and L.tl_page_fork(t, None, None, None, 0, None) == 0 and L.tl_page_fork(t, P + 2, P, P, 1, None) == 3
    assert L.tl_page_compact(t, None, 1, P, P, None) == 1 and L.tl_page_compact(t, P, -1, P, P, None) == 1
    assert L.tl_page_compact(t, P, 1, None, P, None) == 1 and L.tl_page_compact(t, P, 1, P, None, None) == 1 and L.tl_page_compact(t, P, 1, P, P + 2, None) == 3
    for call in (lambda: L.tl_page_reserve(None, P, P, P, P, P, None), lambda: L.tl_page_release(None, P, None),
                 lambda: L.tl_page_fork(None, P, P, P, 1, None), lambda: L.tl_page_compact(None, P, 1, P, P, None)):
        assert call() == 1
    assert L.tl_page_workspace_bytes(t, -1) == 0
    assert L.tl_page_workspace_bytes(t, 0) >= 100 * 20 and L.tl_page_workspace_bytes(t, 10 ** 6) >= 4 * 10 ** 6


def _cache(tl, **kw):
    c = tl.KvCache()
    base = dict(k=P, v=Q, k_scale=P, v_scale=Q, pages=10, format=tl.KV_E2M1, heads=4, head_dim=128, page_tokens=32, k_group=P, v_group=Q)
    for name, value in {**base, **kw}.items():
        setattr(c, name, value)
    return c


@pytest.mark.parametrize("change,status", [
    (dict(k=None), 1), (dict(k_scale=None), 1), (dict(k_group=None), 1), (dict(v_group=None), 1), (dict(head_dim=96), 2),
    (dict(k_group=P + 8), 3), (dict(v_group=Q + 4), 3), (dict(group_page_stride=1032, group_head_stride=256), 3),
    (dict(group_page_stride=1024, group_head_stride=-256), 1), (dict(page_stride=16384, head_stride=4096, token_stride=64), 1),
    (dict(page_stride=16384, head_stride=4096, token_stride=144), 3),            # 72 bytes
    (dict(page_stride=16400, head_stride=4096, token_stride=128), 3),
    (dict(page_stride=2 ** 40, head_stride=128, token_stride=2 ** 27 + 32), 2)])
def test_four_bit_caches_that_are_refused(tl, change, status):
    L, b = tl.lib(), tl.KvBatch()
    for name, value in dict(page_table=P, start=P, token_offsets=P, table_stride=4, requests=2, tokens=6).items():
        setattr(b, name, value)
    c = _cache(tl, **change)
    for call in (L.tl_kv_append, L.tl_kv_read):
        assert call(ctypes.byref(c), ctypes.byref(b), P, Q, 0, 512, None) == status
    assert L.tl_kv_commit(ctypes.byref(c), ctypes.byref(b), P, 4, P, None, None) == status
    assert L.tl_tree_attention(ctypes.byref(c), ctypes.byref(b), P, 1024, 8, None, 0, 0.1, Q, 1024, None, None) == status
    assert L.tl_page_copy(ctypes.byref(c), ctypes.byref(c), P, P, 3, None) == status
    good = _cache(tl)
    assert L.tl_page_copy(ctypes.byref(good), ctypes.byref(c), P, P, 3, None) == status


def test_copy_arguments(tl):
    L, c = tl.lib(), _cache(tl)
    copy = lambda to, moves=P, n=P, most=3: L.tl_page_copy(ctypes.byref(c), ctypes.byref(to), moves, n, most, None)  # noqa: E731
    for change in (dict(format=tl.KV_INT8), dict(heads=5), dict(head_dim=64), dict(page_tokens=64)):
        assert copy(_cache(tl, **change)) == 1
    assert copy(c, moves=None) == 1 and copy(c, most=-1) == 1 and copy(c, moves=P + 2) == 3 and copy(c, n=P + 1) == 3 and copy(c, most=0) == 0
    assert L.tl_page_copy(None, ctypes.byref(c), P, P, 3, None) == 1 and L.tl_page_copy(ctypes.byref(c), None, P, P, 3, None) == 1
