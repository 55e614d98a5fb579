"""Rotary positions without a GPU: the frequencies, and what the entry points refuse before any CUDA call."""
import ctypes
import math
from decimal import Decimal, getcontext

import pytest

P, Q = 0x10000, 0x900000
getcontext().prec = 60
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.fixture(scope="module")
def tl():
    from paper_2607_04031_b200 import build
    build.build()
    from paper_2607_04031_b200 import binding
    return binding


def _frequencies(dim, base, kind, factor, original, low, high):
    base, factor, original, low, high = (Decimal(v) for v in (base, factor, original, low, high))
    clamp = lambda v: min(max(v, Decimal(0)), Decimal(1))  # noqa: E731
    out = []
    if kind == 3:
        pair = lambda n: dim * (original / (n * 2 * PI)).ln() / (2 * base.ln())  # noqa: E731
        lo = max(Decimal(math.floor(pair(high))), Decimal(0))
        hi = min(Decimal(math.ceil(pair(low))), Decimal(dim - 1))
        hi = lo + Decimal("0.001") if hi <= lo else hi
    for i in range(dim // 2):
        f = (-base.ln() * 2 * i / dim).exp()
        if kind == 1:
            f /= factor
        if kind == 2:
            u = clamp((original * f / (2 * PI) - low) / (high - low))
            f = (1 - u) * f / factor + u * f
        if kind == 3:
            u = clamp((i - lo) / (hi - lo))
            f = u * f / factor + (1 - u) * f
        out.append(f)
    return out


@pytest.mark.parametrize("dim,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (48, 1e6), (1024, 1.5)])
@pytest.mark.parametrize("kind,factor,original,low,high", [(0, 1.0, 0.0, 1.0, 4.0), (1, 4.0, 0.0, 1.0, 4.0), (2, 8.0, 8192.0, 1.0, 4.0),
                                                           (3, 32.0, 4096.0, 1.0, 32.0), (3, 2.0, 64.0, 30.0, 30.5), (2, 1.0, 100.0, 0.5, 9.0)])
def test_turns_are_the_formula_to_their_last_bits(tl, dim, base, kind, factor, original, low, high):
    got = [w & (2 ** 64 - 1) for w in tl.rope_turns(dim, base, kind, factor, original, low, high).tolist()]
    for w, f in zip(got, _frequencies(dim, base, kind, factor, original, low, high)):
        want = f / (2 * PI) * 2 ** 64
        # long double: a few roundings of 2^-64 each, and the base's power (half a unit times the logarithm's size, at most 2^4)
        assert abs(Decimal(w) - want) <= Decimal(1) + want * Decimal(2) ** -58


@pytest.mark.parametrize("args", [(0, 1e4, 0, 1, 0, 1, 4), (7, 1e4, 0, 1, 0, 1, 4), (1026, 1e4, 0, 1, 0, 1, 4), (8, 1.0, 0, 1, 0, 1, 4),
                                  (8, math.inf, 0, 1, 0, 1, 4), (8, math.nan, 0, 1, 0, 1, 4), (8, 1e4, 4, 1, 0, 1, 4), (8, 1e4, -1, 1, 0, 1, 4),
                                  (8, 1e4, 1, 0.5, 0, 1, 4), (8, 1e4, 1, math.nan, 0, 1, 4), (8, 1e4, 2, 8, 0, 1, 4), (8, 1e4, 2, 8, 100, 4, 4),
                                  (8, 1e4, 3, 8, 100, 0, 4), (8, 1e4, 3, 8, math.inf, 1, 4), (8, 1e4, 3, 8, 100, 1, math.inf)])
def test_turns_refused(tl, args):
    out = (ctypes.c_uint64 * 600)()
    assert tl.lib().tl_rope_turns(*args, ctypes.addressof(out)) == 1
    assert tl.lib().tl_rope_turns(8, 1e4, 0, 1, 0, 1, 4, None) == 1


def _rope(tl, **kw):
    r = tl.Rope()
    for name, value in {**dict(turns=P, amplitude=1.0, rotary_dim=128, layout=0), **kw}.items():
        setattr(r, name, value)
    return r


ROPES = [(dict(turns=None), 1), (dict(amplitude=math.inf), 1), (dict(amplitude=math.nan), 1), (dict(rotary_dim=0), 1), (dict(rotary_dim=3), 1),
         (dict(rotary_dim=130), 1), (dict(layout=2), 1), (dict(layout=-1), 1), (dict(turns=P + 4), 3)]


def _rows(tl, rope=None, x=P, xs=512, out=Q, os_=512, elem=0, tokens=3, heads=4, dim=128, pos=P, inverse=0):
    r = rope or _rope(tl)
    return tl.lib().tl_rope_rows(ctypes.byref(r), x, xs, out, os_, elem, tokens, heads, dim, pos, inverse, None)


def _append(tl, rope=None, positions=None, q=P, qs=1024, heads=8, out=Q, os_=1024, k=P, v=Q, elem=0, stride=512, tokens=6, fmt=2):
    c, b, r = tl.KvCache(), tl.KvBatch(), rope or _rope(tl)
    for name, value in dict(k=P, v=Q, k_scale=P, v_scale=Q, pages=10, format=fmt, heads=4, head_dim=128, page_tokens=32).items():
        setattr(c, name, value)
    for name, value in dict(page_table=P, start=P, token_offsets=P, table_stride=4, requests=2, tokens=tokens).items():
        setattr(b, name, value)
    return tl.lib().tl_rope_append(ctypes.byref(c), ctypes.byref(b), ctypes.byref(r), positions, q, qs, heads, out, os_, k, v, elem, stride, None)


@pytest.mark.parametrize("change,status", ROPES)
def test_rope_descriptions_that_are_refused(tl, change, status):
    assert _rows(tl, _rope(tl, **change)) == status
    assert _append(tl, _rope(tl, **change)) == status


def test_rows_arguments(tl):
    assert _rows(tl, x=None) == 1 and _rows(tl, out=None) == 1 and _rows(tl, pos=None) == 1 and _rows(tl, elem=2) == 1
    assert _rows(tl, xs=511) == 1 and _rows(tl, os_=511) == 1 and _rows(tl, tokens=-1) == 1 and _rows(tl, heads=-1) == 1
    assert _rows(tl, dim=127) == 1 and _rows(tl, dim=126) == 1 and _rows(tl, dim=1026) == 2 and _rows(tl, dim=0) == 1
    assert _rows(tl, out=P, os_=520) == 1                                            # in place, with another stride
    assert _rows(tl, x=P + 1) == 3 and _rows(tl, out=Q + 1) == 3 and _rows(tl, pos=P + 2) == 3 and _rows(tl, x=P + 2, elem=1) == 3
    assert _rows(tl, xs=2 ** 41) == 2
    assert _rows(tl, tokens=0) == 0 and _rows(tl, heads=0) == 0
    assert tl.lib().tl_rope_rows(None, P, 512, Q, 512, 0, 3, 4, 128, P, 0, None) == 1


def test_append_arguments(tl):
    assert _append(tl, q=None) == 1 and _append(tl, out=None) == 1 and _append(tl, heads=0) == 1 and _append(tl, heads=-1) == 1
    assert _append(tl, k=None) == 1 and _append(tl, v=None) == 1 and _append(tl, elem=2) == 1 and _append(tl, stride=511) == 1
    assert _append(tl, qs=1023) == 1 and _append(tl, os_=1016) == 1
    assert _append(tl, out=P, elem=1) == 1 and _append(tl, out=P, os_=1032) == 1     # in place: bf16, one stride
    assert _append(tl, q=P + 8) == 3 and _append(tl, out=Q + 8) == 3 and _append(tl, k=P + 8) == 3 and _append(tl, qs=1028) == 3
    assert _append(tl, os_=1028) == 3 and _append(tl, stride=516) == 3 and _append(tl, positions=P + 2) == 3
    assert _append(tl, fmt=3) == 1 and _append(tl, tokens=-1) == 1 and _append(tl, tokens=0) == 0


def test_positions_arguments(tl):
    call = lambda *a: tl.lib().tl_tree_positions(*a, None)  # noqa: E731
    assert call(None, P, P, 1, 4, P) == 1 and call(P, None, P, 1, 4, P) == 1 and call(P, P, None, 1, 4, P) == 1 and call(P, P, P, 1, 4, None) == 1
    assert call(P, P, P, -1, 4, P) == 1 and call(P, P, P, 1, -4, P) == 1 and call(P, P, P, 0, 4, P) == 0 and call(P, P, P + 2, 1, 4, P) == 3
