"""What the binding passes on and refuses, without a GPU: stand-ins for device tensors, calls that end before any CUDA call."""
import pytest
import torch


class Device:
    def __init__(self, index):
        self.type, self.index = "cuda", index


class OnDevice:
    """A CPU tensor that says it lies on a device: shapes, strides and types are the tensor's own."""
    is_cuda = True

    def __init__(self, t, index=0):
        self.t, self.device, self.shape, self.dtype = t, Device(index), t.shape, t.dtype

    def stride(self, *a):
        return self.t.stride(*a)

    def dim(self):
        return self.t.dim()

    def is_contiguous(self):
        return self.t.is_contiguous()

    def get_device(self):
        return self.device.index

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
