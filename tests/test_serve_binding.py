"""What the binding of rotary positions, pages and the 4-bit cache passes on and refuses, without a GPU."""
import pytest
import torch

from test_kv_binding import OnDevice, Stream, no_library, tl  # noqa: F401  (fixtures)

I32, B16, F32, E4M3 = torch.int32, torch.bfloat16, torch.float32, torch.float8_e4m3fn


def _calls(tl, index=None, stream=Stream):
    """Every call by the names of its tensors; index: where each lies."""
    index = index or {}
    at = lambda name, *shape, dtype=I32: OnDevice(torch.zeros(*shape, dtype=dtype), index.get(name, 0))  # noqa: E731
    four = lambda: tl.kv_cache(at("kc", 3, 2, 16, 32, dtype=torch.uint8), at("vc", 3, 2, 16, 32, dtype=torch.uint8), at("ks", 3, 2, 16, dtype=F32),  # noqa: E731
                               at("vs", 3, 2, 16, dtype=F32), at("kg", 3, 2, 16, 4, dtype=E4M3), at("vg", 3, 2, 16, 4, dtype=E4M3))
    batch = lambda: tl.kv_batch(at("table", 1, 4), at("start", 1), at("offsets", 2), 5)  # noqa: E731
    rope = lambda: tl.rope(at("turns", 32, dtype=torch.int64))  # noqa: E731
    tables = lambda: tl.page_tables(at("table", 2, 4), at("held", 2), at("holders", 9), 16)  # noqa: E731
    return {
        "rows": lambda: tl.rope_rows(rope(), at("x", 5, 2, 64, dtype=B16), at("out", 5, 2, 64, dtype=B16), at("positions", 5), stream=stream),
        "append": lambda: tl.rope_append(four(), batch(), rope(), at("q", 5, 4, 64, dtype=B16), at("out", 5, 4, 64, dtype=B16),
                                         at("k", 5, 2, 64, dtype=B16), at("v", 5, 2, 64, dtype=B16), at("positions", 5), stream=stream),
        "positions": lambda: tl.tree_positions(at("parents", 5), at("offsets", 2), at("start", 1), at("positions", 5), stream=stream),
        "reserve": lambda: tl.page_reserve(tables(), at("start", 2), at("tokens", 2), at("moves", 2, 3), at("n", 1), at("missing", 1), stream=stream),
        "release": lambda: tl.page_release(tables(), at("tokens", 2), stream=stream),
        "fork": lambda: tl.page_fork(tables(), at("from", 1), at("to", 1), at("tokens", 1), stream=stream),
        "compact": lambda: tl.page_compact(tables(), at("moves", 4, 3), at("n", 1), at("in_use", 1), stream=stream),
        "copy": lambda: tl.page_copy(four(), at("moves", 4, 3), at("n", 1), stream=stream)}


TENSORS = {"rows": "turns x out positions", "append": "kc vc ks vs kg vg table start offsets turns q out k v positions",
           "positions": "parents offsets start positions", "reserve": "table held holders start tokens moves n missing",
           "release": "table held holders tokens", "fork": "table held holders from to tokens", "compact": "table held holders moves n in_use",
           "copy": "kc vc ks vs kg vg moves n"}


def test_calls_on_one_device_go_through(no_library):  # noqa: F811
    for call in _calls(no_library).values():
        call()


@pytest.mark.parametrize("call,name", [(c, n) for c, names in TENSORS.items() for n in names.split()])
def test_a_tensor_on_another_device_is_refused(no_library, call, name):  # noqa: F811
    with pytest.raises(ValueError, match="cuda:"):
        _calls(no_library, {name: 1})[call]()


@pytest.mark.parametrize("call", list(TENSORS))
@pytest.mark.parametrize("current", [0, 1])
def test_the_current_device_has_to_be_the_tensors(no_library, monkeypatch, call, current):  # noqa: F811
    monkeypatch.setattr(no_library, "_current_device", lambda: current)
    monkeypatch.setattr(no_library, "_current_stream", lambda device: 0)
    run = _calls(no_library, stream=None)[call]
    if current == 0:
        run()
    else:
        with pytest.raises(ValueError, match="cuda:"):
            run()


def _z(*shape, dtype=I32):
    return OnDevice(torch.zeros(*shape, dtype=dtype))


def test_four_bit_caches_that_are_refused(tl):  # noqa: F811
    k, s, g = lambda: _z(3, 2, 16, 32, dtype=torch.uint8), lambda: _z(3, 2, 16, dtype=F32), lambda *n: _z(*(n or (3, 2, 16, 4)), dtype=E4M3)  # noqa: E731
    c = tl.kv_cache(k(), k(), s(), s(), g(), g())
    assert (c.format, c.head_dim, c.token_stride, c.group_head_stride) == (tl.KV_E2M1, 64, 64, 64)
    for args in ((k(), k(), s(), s()), (k(), k(), s(), s(), g(), None), (k(), k(), None, None, g(), g()), (k(), k(), s(), s(), g(3, 2, 16, 2), g(3, 2, 16, 2)),
                 (k(), k(), s(), s(), _z(3, 2, 16, 4, dtype=torch.uint8), g()), (k(), k(), s(), s(), OnDevice(g().transpose(1, 2).contiguous().transpose(1, 2)), g())):
        with pytest.raises(ValueError):
            tl.kv_cache(*args)
    i8 = lambda: _z(3, 2, 16, 64, dtype=torch.int8)  # noqa: E731
    with pytest.raises(ValueError, match="group"):
        tl.kv_cache(i8(), i8(), s(), s(), g(), g())


def test_shapes_and_types_that_are_refused(no_library):  # noqa: F811
    t = no_library
    r, tables = t.rope(_z(32, dtype=torch.int64)), t.page_tables(_z(2, 4), _z(2), _z(9), 16)
    x, p = _z(5, 2, 64, dtype=B16), _z(5)
    for f in (lambda: t.rope(_z(32)), lambda: t.rope_rows(r, x, _z(5, 2, 64, dtype=F32), p), lambda: t.rope_rows(r, x, _z(5, 3, 64, dtype=B16), p),
              lambda: t.rope_rows(r, x, x, _z(4)), lambda: t.rope_rows(r, x, x, _z(5, dtype=torch.int64)),
              lambda: t.rope_rows(r, OnDevice(x.transpose(0, 1)), OnDevice(x.transpose(0, 1)), _z(2)), lambda: t.rope_rows(r, _z(5, 64, dtype=B16), _z(5, 64, dtype=B16), p),
              lambda: t.page_tables(_z(2, 4), _z(3), _z(9), 16), lambda: t.page_tables(_z(2, 4), _z(2), _z(9, dtype=torch.int64), 16),
              lambda: t.page_reserve(tables, _z(2), _z(2), _z(1, 3), _z(1), _z(1)), lambda: t.page_reserve(tables, _z(2), _z(3), _z(2, 3), _z(1), _z(1)),
              lambda: t.page_reserve(tables, _z(2), _z(2), _z(2, 2), _z(1), _z(1)), lambda: t.page_fork(tables, _z(1), _z(2), _z(1)),
              lambda: t.page_compact(tables, _z(12), _z(1), _z(1)), lambda: t.page_release(tables, _z(3))):
        with pytest.raises(ValueError):
            f()


def test_the_library_refuses_what_shares_memory(tl):  # noqa: F811
    """Rows that overlap, or an output that lies over its input with another stride."""
    r = tl.rope(_z(32, dtype=torch.int64))
    shared = OnDevice(torch.zeros(6 * 128, dtype=B16).as_strided((5, 2, 64), (64, 64, 1)))
    with pytest.raises(tl.TileLensError) as e:
        tl.rope_rows(r, shared, _z(5, 2, 64, dtype=B16), _z(5), stream=Stream)
    assert e.value.status == 1
    wide = torch.zeros(5, 200, dtype=B16)
    with pytest.raises(tl.TileLensError) as e:
        tl.rope_rows(r, OnDevice(wide[:, :128].unflatten(1, (2, 64))), _z(5, 2, 64, dtype=B16), _z(5), stream=Stream)
    assert e.value.status == 1                                # (stand-ins all lie at one address: in place, two strides)
