"""Refusals of the key/value cache, attention and verification entry points (CPU only: they return before any CUDA call)."""
import ctypes
import math

import pytest

P, Q = 0x10000, 0x900000


@pytest.fixture(scope="module")
def tl():
    from paper_2607_04031_b200 import build
    build.build()
    from paper_2607_04031_b200 import binding
    return binding


def _cache(tl, **kw):
    c = tl.KvCache()
    base = dict(k=P, v=Q, k_scale=P, v_scale=Q, pages=10, format=tl.KV_INT8, heads=4, head_dim=128, page_tokens=32)
    for name, value in {**base, **kw}.items():
        setattr(c, name, value)
    return c


def _batch(tl, **kw):
    b = tl.KvBatch()
    for name, value in {**dict(page_table=P, start=P, token_offsets=P, table_stride=4, requests=2, tokens=6), **kw}.items():
        setattr(b, name, value)
    return b


def _append(tl, cache=None, batch=None, k=P, v=Q, elem=0, stride=512):
    c, b = cache or _cache(tl), batch or _batch(tl)
    return tl.lib().tl_kv_append(ctypes.byref(c), ctypes.byref(b), k, v, elem, stride, None)


def _attend(tl, cache=None, batch=None, q=P, q_stride=1024, heads=8, mask=None, words=0, scale=0.1, out=Q, out_stride=1024, lse=None):
    c, b = cache or _cache(tl), batch or _batch(tl)
    return tl.lib().tl_tree_attention(ctypes.byref(c), ctypes.byref(b), q, q_stride, heads, mask, words, scale, out, out_stride, lse, None)


CACHES = [
    (dict(k=None), 1), (dict(v=None), 1), (dict(k_scale=None), 1), (dict(v_scale=None), 1), (dict(pages=0), 1),
    (dict(heads=0), 1), (dict(head_dim=0), 1), (dict(format=3), 1), (dict(format=-1), 1), (dict(page_tokens=0), 1),
    (dict(head_dim=96), 2), (dict(head_dim=80), 2), (dict(page_tokens=8), 2), (dict(page_tokens=48), 2), (dict(page_tokens=2048), 2),
    (dict(k=P + 8), 3), (dict(v=Q + 4), 3), (dict(k_scale=P + 4), 3),
    (dict(page_stride=16384, head_stride=4096, token_stride=64), 1),                # rows overlap
    (dict(page_stride=16384, head_stride=4096, token_stride=132), 3),
    (dict(page_stride=16392, head_stride=4096, token_stride=128), 3),
    (dict(page_stride=-16384, head_stride=4096, token_stride=128), 1),
    (dict(scale_page_stride=130, scale_head_stride=32), 3), (dict(scale_page_stride=128, scale_head_stride=-32), 1),
]


@pytest.mark.parametrize("change,status", CACHES)
def test_cache_descriptions_that_are_refused(tl, change, status):
    assert _append(tl, _cache(tl, **change)) == status
    assert _attend(tl, _cache(tl, **change)) == status
    c, b = _cache(tl, **change), _batch(tl)
    assert tl.lib().tl_kv_commit(ctypes.byref(c), ctypes.byref(b), P, 4, P, None, None) == status
    assert tl.lib().tl_tree_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(b), 8) == 0


@pytest.mark.parametrize("change,status", [(dict(page_table=None), 1), (dict(start=None), 1), (dict(token_offsets=None), 1),
                                           (dict(table_stride=0), 1), (dict(requests=-1), 1), (dict(tokens=-1), 1),
                                           (dict(page_table=P + 2), 3)])
def test_batch_descriptions_that_are_refused(tl, change, status):
    assert _append(tl, batch=_batch(tl, **change)) == status
    assert _attend(tl, batch=_batch(tl, **change)) == status


def test_append_and_read_arguments(tl):
    assert _append(tl, k=None) == 1 and _append(tl, v=None) == 1 and _append(tl, elem=2) == 1
    assert _append(tl, stride=511) == 1 and _append(tl, stride=516) == 3 and _append(tl, k=P + 8) == 3
    assert _append(tl, batch=_batch(tl, tokens=0)) == 0 and _append(tl, batch=_batch(tl, requests=0)) == 0
    c, b = _cache(tl), _batch(tl)
    assert tl.lib().tl_kv_read(ctypes.byref(c), ctypes.byref(b), None, Q, 0, 512, None) == 1
    assert tl.lib().tl_kv_read(None, ctypes.byref(b), P, Q, 0, 512, None) == 1
    assert tl.lib().tl_kv_read(ctypes.byref(c), None, P, Q, 0, 512, None) == 1


def test_commit_and_mask_arguments(tl):
    c, b = _cache(tl), _batch(tl)
    call = lambda acc=P, stride=4, n=P: tl.lib().tl_kv_commit(ctypes.byref(c), ctypes.byref(b), acc, stride, n, None, None)  # noqa: E731
    assert call(acc=None) == 1 and call(stride=0) == 1 and call(n=None) == 1
    mask = lambda *a: tl.lib().tl_tree_mask(*a, None)  # noqa: E731
    assert mask(None, P, 1, 4, P, 1) == 1 and mask(P, None, 1, 4, P, 1) == 1 and mask(P, P, 1, 4, None, 1) == 1
    assert mask(P, P, 1, 4, P, 0) == 1 and mask(P, P, -1, 4, P, 1) == 1 and mask(P, P, 1, 0, P, 1) == 0


def test_attention_arguments(tl):
    assert _attend(tl, heads=6) == 1 and _attend(tl, heads=0) == 1                   # not a multiple of the cache's heads
    assert _attend(tl, q=None) == 1 and _attend(tl, out=None) == 1
    assert _attend(tl, q_stride=1023) == 1 and _attend(tl, out_stride=1000) == 1
    assert _attend(tl, q_stride=1028) == 3 and _attend(tl, q=P + 8) == 3 and _attend(tl, out=Q + 2) == 3
    assert _attend(tl, mask=P, words=0) == 1
    assert _attend(tl, scale=math.inf) == 1 and _attend(tl, scale=math.nan) == 1
    assert _attend(tl, batch=_batch(tl, tokens=2 ** 30)) == 2
    assert _attend(tl, batch=_batch(tl, tokens=0)) == 0


def test_verify_arguments(tl):
    def call(**kw):
        a = {**dict(target=P, ts=100, draft=P, ds=100, vocab=100, tokens=P, parents=P, offs=P, requests=2, rows=6, accept=P,
                    sample=P, acc=P, stride=4, n=P, nxt=P), **kw}
        return tl.lib().tl_tree_verify(a["target"], a["ts"], a["draft"], a["ds"], a["vocab"], a["tokens"], a["parents"], a["offs"],
                                       a["requests"], a["rows"], a["accept"], a["sample"], a["acc"], a["stride"], a["n"], a["nxt"], None)
    for name in ("target", "tokens", "parents", "offs", "accept", "sample", "acc", "n", "nxt"):
        assert call(**{name: None}) == 1, name
    assert call(ts=99) == 1 and call(ds=99) == 1 and call(vocab=0) == 1 and call(stride=0) == 1 and call(vocab=2 ** 31) == 1
    assert call(requests=-1) == 1 and call(rows=-1) == 1 and call(requests=0) == 0


def test_binding_refuses_wrong_tensors(tl):
    import torch
    with pytest.raises(ValueError, match="CUDA|expected"):
        tl.kv_cache(torch.zeros(1, 1, 16, 64, dtype=torch.int8), torch.zeros(1, 1, 16, 64, dtype=torch.int8))


def test_tokens_further_apart_than_32_bit_offsets_allow_are_refused(tl):
    # INT8: 2^26 bytes between tokens are the most; bf16: 2^25 elements
    for fmt, most in ((tl.KV_INT8, 2 ** 26), (tl.KV_BF16, 2 ** 25)):
        wide = dict(format=fmt, page_stride=64 * most, head_stride=128, token_stride=most + 16)
        assert _append(tl, _cache(tl, **wide)) == 2 and _attend(tl, _cache(tl, **wide)) == 2


def test_pointers_off_their_elements_are_refused(tl):
    # every array these calls read or write in words of four bytes: two bytes off it would be a misaligned access
    names = ("target", "draft", "tokens", "parents", "offs", "accept", "sample", "acc", "n", "nxt")
    for name in names:
        a = {**{k: P for k in names}, name: P + 2}
        assert tl.lib().tl_tree_verify(a["target"], 100, a["draft"], 100, 100, a["tokens"], a["parents"], a["offs"], 2, 6, a["accept"],
                                       a["sample"], a["acc"], 4, a["n"], a["nxt"], None) == 3, name
    for i in range(3):
        a = [P + 2 * (k == i) for k in range(3)]
        assert tl.lib().tl_tree_mask(a[0], a[1], 1, 4, a[2], 1, None) == 3
        c, b = _cache(tl), _batch(tl)
        assert tl.lib().tl_kv_commit(ctypes.byref(c), ctypes.byref(b), a[0], 4, a[1], a[2], None) == 3
