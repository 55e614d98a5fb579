"""Descriptions of caches, batches, frequencies and page tables keep their tensors as long as they live, and no longer."""
import gc
import weakref

import pytest
import torch

from test_kv_binding import OnDevice, tl  # noqa: F401  (fixture)

I32, E4M3 = torch.int32, torch.float8_e4m3fn


def _at(*shape, dtype=I32):
    return OnDevice(torch.zeros(*shape, dtype=dtype))


def _u8():
    return _at(3, 2, 16, 32, dtype=torch.uint8)


MAKE = {
    "kv_cache": lambda tl: (tl.kv_cache, [_u8(), _u8(), *(_at(3, 2, 16, dtype=torch.float32) for _ in range(2)), *(_at(3, 2, 16, 4, dtype=E4M3) for _ in range(2))], ()),
    "kv_batch": lambda tl: (tl.kv_batch, [_at(1, 4), _at(1), _at(2)], (5,)),
    "rope": lambda tl: (tl.rope, [_at(32, dtype=torch.int64)], ()),
    "page_tables": lambda tl: (tl.page_tables, [_at(2, 4), _at(2), _at(9)], (16,)),
}


@pytest.mark.parametrize("what", list(MAKE))
def test_tensors_go_with_the_last_reference(tl, what):  # noqa: F811
    make, tensors, rest = MAKE[what](tl)
    watch = [weakref.ref(t) for t in tensors]
    gc.collect()
    gc.disable()                                             # (a pool must not wait for the collector)
    try:
        d = make(*tensors, *rest)
        del tensors
        assert all(w() is not None for w in watch)
        del d
        assert all(w() is None for w in watch)
    finally:
        gc.enable()
