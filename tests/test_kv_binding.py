"""What the binding passes on and refuses, without a GPU: stand-ins for device tensors, calls that end before any CUDA call."""
import pytest
import torch


class Device:
    def __init__(self, index):
        self.type, self.index = "cuda", index


class OnDevice(torch.Tensor):
    """A CPU tensor that says it lies on a device: shapes, strides and types are the tensor's own."""
    is_cuda = True

    def __new__(cls, t, index=0):
        self = torch.Tensor._make_subclass(cls, t)
        self.index = index
        return self

    @property
    def device(self):
        return Device(self.index)

    def get_device(self):
        return self.index

    def data_ptr(self):
        return 0x10000


class Stream:
    cuda_stream = 0


@pytest.fixture()
def tl():
    from paper_2607_04031_b200 import build
    build.build()
    from paper_2607_04031_b200 import binding
    return binding


def _verify(tl, target, draft):
    rows = target.shape[0]
    i32 = lambda *shape: OnDevice(torch.zeros(*shape, dtype=torch.int32))  # noqa: E731
    tl.tree_verify(OnDevice(target), None if draft is None else OnDevice(draft), i32(rows), i32(rows), i32(2),
                   OnDevice(torch.zeros(rows)), OnDevice(torch.zeros(1)), i32(1, 4), i32(1), i32(1), stream=Stream)


@pytest.mark.parametrize("which", ["target", "draft"])
@pytest.mark.parametrize("stride", [0, 1, 99])
def test_verify_refuses_rows_that_share_memory(tl, which, stride):
    # one distribution for several rows, or rows that overlap: read with a longer stride they would be read past their end
    apart = torch.zeros(6, 100)
    shared = torch.zeros(6 * 100).as_strided((6, 100), (stride, 1))
    with pytest.raises(tl.TileLensError) as e:
        _verify(tl, shared if which == "target" else apart, shared if which == "draft" else apart)
    assert e.value.status == 1


def _cache(tl, **index):
    at = lambda name, *shape, dtype=torch.float32: OnDevice(torch.zeros(*shape, dtype=dtype), index.get(name, 0))  # noqa: E731
    return tl.kv_cache(at("k", 3, 2, 16, 64, dtype=torch.int8), at("v", 3, 2, 16, 64, dtype=torch.int8), at("ks", 3, 2, 16), at("vs", 3, 2, 16))


def _batch(tl, **index):
    at = lambda name, *shape: OnDevice(torch.zeros(*shape, dtype=torch.int32), index.get(name, 0))  # noqa: E731
    return tl.kv_batch(at("table", 1, 4), at("start", 1), at("offsets", 2), 5)


def _calls(tl, cache, batch, index=None, stream=Stream):
    """Every call of a step by the names of its tensors; index: where each lies."""
    index = index or {}
    at = lambda name, *shape, dtype=torch.int32: OnDevice(torch.zeros(*shape, dtype=dtype), index.get(name, 0))  # noqa: E731
    f32, b16 = torch.float32, torch.bfloat16
    return {
        "append": lambda: tl.kv_append(cache, batch, at("k", 5, 2, 64, dtype=b16), at("v", 5, 2, 64, dtype=b16), stream=stream),
        "read": lambda: tl.kv_read(cache, batch, at("k", 5, 2, 64, dtype=f32), at("v", 5, 2, 64, dtype=f32), stream=stream),
        "commit": lambda: tl.kv_commit(cache, batch, at("accepted", 1, 3), at("n", 1), at("new", 1), stream=stream),
        "mask": lambda: tl.tree_mask(at("parents", 5), at("offsets", 2), at("mask", 5, 1), stream=stream),
        "attention": lambda: tl.tree_attention(cache, batch, at("q", 5, 4, 64, dtype=b16), at("out", 5, 4, 64, dtype=b16), at("mask", 5, 1),
                                               None, at("lse", 5, 4, dtype=f32), stream=stream),
        "verify": lambda: tl.tree_verify(at("target", 5, 9, dtype=f32), at("draft", 5, 9, dtype=f32), at("tokens", 5), at("parents", 5),
                                         at("offsets", 2), at("accept", 5, dtype=f32), at("sample", 1, dtype=f32), at("accepted", 1, 3),
                                         at("n", 1), at("next", 1), stream=stream)}


TENSORS = {"append": "k v", "read": "k v", "commit": "accepted n new", "mask": "parents offsets mask", "attention": "q out mask lse",
           "verify": "target draft tokens parents offsets accept sample accepted n next"}


@pytest.fixture()
def no_library(tl, monkeypatch):
    """What reaches the library counts as done."""
    class Library:
        def __getattr__(self, name):
            return lambda *a: 0
    monkeypatch.setattr(tl, "lib", lambda: Library())
    return tl


def test_a_step_on_one_device_goes_through(no_library):
    for call in _calls(no_library, _cache(no_library), _batch(no_library)).values():
        call()


@pytest.mark.parametrize("call,name", [(c, n) for c, names in TENSORS.items() for n in names.split()])
def test_a_tensor_on_another_device_is_refused(no_library, call, name):
    with pytest.raises(ValueError, match="cuda:"):
        _calls(no_library, _cache(no_library), _batch(no_library), {name: 1})[call]()


@pytest.mark.parametrize("name", ["k", "v", "ks", "vs"])
def test_a_cache_on_two_devices_is_refused(no_library, name):
    with pytest.raises(ValueError, match="cuda:"):
        _cache(no_library, **{name: 1})


@pytest.mark.parametrize("name", ["table", "start", "offsets"])
def test_a_batch_on_two_devices_is_refused(no_library, name):
    with pytest.raises(ValueError, match="cuda:"):
        _batch(no_library, **{name: 1})


@pytest.mark.parametrize("call", ["append", "read", "commit", "attention"])
def test_a_batch_beside_another_devices_cache_is_refused(no_library, call):
    away = _batch(no_library, table=1, start=1, offsets=1)
    with pytest.raises(ValueError, match="cuda:"):
        _calls(no_library, _cache(no_library), away)[call]()


@pytest.mark.parametrize("call", list(TENSORS))
@pytest.mark.parametrize("current", [0, 1])
def test_the_current_device_has_to_be_the_tensors(no_library, monkeypatch, call, current):
    # the library launches on the current device: another one's stream would not do
    monkeypatch.setattr(no_library, "_current_device", lambda: current)
    monkeypatch.setattr(no_library, "_current_stream", lambda device: 0)
    run = _calls(no_library, _cache(no_library), _batch(no_library), stream=None)[call]
    if current == 0:
        run()
    else:
        with pytest.raises(ValueError, match="cuda:"):
            run()
