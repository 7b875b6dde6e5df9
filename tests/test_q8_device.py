"""The 8-bit calls launch on the current device's stream: tensors of another device are refused before anything is launched.  With
stand-ins for the tensors, the library and the current device, so that no GPU is needed (nor a second one)."""
import os

import pytest
import torch

from paper_2507_17301_amd import binding as nm

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_17301_amd", "libnmconv.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libnmconv.so not built (python -m paper_2507_17301_amd.build)")


class Tensor:
    """A contiguous tensor on a device that need not exist."""
    is_cuda = True

    def __init__(self, shape, dtype, device):
        self.shape, self.dtype, self.device_index = torch.Size(shape), dtype, device

    def get_device(self):
        return self.device_index

    def dim(self):
        return len(self.shape)

    def stride(self):
        return (self.shape[1], 1) if len(self.shape) == 2 else (1,)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


class Library:
    """Counts the calls that would launch."""
    launches = 0

    def __getattr__(self, name):
        def call(*args):
            self.launches += 1
            return nm.NM_OK
        return call


@pytest.fixture
def machine(monkeypatch):
    """Two devices, of which number 0 is the current one."""
    nm.lib()
    library = Library()
    monkeypatch.setattr(nm, "_lib", library)
    monkeypatch.setattr(nm._torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(nm._torch._C, "_cuda_getCurrentRawStream", lambda device: 0)
    return library


def _calls(dev):
    f32, i8 = torch.float32, torch.int8
    x, y, r, out = (Tensor((3, 32), f32, dev) for _ in range(4))
    q, s = Tensor((3, 32), i8, dev), Tensor((3,), f32, dev)
    w, ws = Tensor((32, 32), i8, dev), Tensor((32,), f32, dev)
    packed = nm.Q8Weights(None, 32, 32, False)
    return {"quantize": lambda: nm.nm_quantize_q8(x, q, s),
            "rmsnorm": lambda: nm.nm_rmsnorm_q8(x, None, r, q=q, scales=s, residual_out=out),
            "dequantize": lambda: nm.nm_dequantize_q8(q, s, y=y),
            "pack": lambda: nm.nm_q8_pack(w, ws),
            "linear": lambda: nm.nm_linear_q8(q, s, packed, y=y)}


@pytest.mark.parametrize("name", sorted(_calls(0)))
def test_tensors_of_another_device_are_refused(machine, name):
    with pytest.raises(ValueError, match="device 1"):
        _calls(1)[name]()
    assert machine.launches == 0
    _calls(0)[name]()
    assert machine.launches == 1
