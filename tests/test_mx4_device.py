"""The calls in MX4 and those for experts launch on the current device's stream: tensors of another device are refused before anything
is launched.  With stand-ins for the tensors, the library and the current device, so that no GPU is needed (nor a second one)."""
import pytest
import torch

from paper_2507_17301_amd import binding as nm
from paper_2507_17301_amd.feedforward import ExpertsMX4, FeedForwardMX4
from test_q8_device import Tensor, machine, pytestmark  # noqa: F401  (the fixture and the mark)


class Made(Tensor):
    """A stand-in that also makes tensors, as the routing's outputs are made."""

    def new_empty(self, shape, dtype):
        return Made((shape,) if isinstance(shape, int) else shape, dtype, self.device_index)

    def unbind(self):
        return [Made(self.shape[1:], self.dtype, self.device_index) for _ in range(self.shape[0])]

    def view(self, dtype):
        return Made(self.shape, dtype, self.device_index)

    def split_with_sizes(self, sizes):
        return [Made((n,), self.dtype, self.device_index) for n in sizes]


def _calls(dev):
    f32, u8, i32 = torch.float32, torch.uint8, torch.int32
    x, r, out = (Tensor((3, 64), f32, dev) for _ in range(3))
    q, s, yq, ys = Tensor((3, 32), u8, dev), Tensor((3, 2), u8, dev), Tensor((3, 32), u8, dev), Tensor((3, 2), u8, dev)
    packed, several = nm.MX4Weights(None, 1, 64, 64, False), nm.MX4Weights(None, 2, 64, 64, False)
    offsets, rows = Tensor((3,), i32, dev), Tensor((3,), i32, dev)
    return {"quantize": lambda: nm.nm_quantize_mx4(x, q, s),
            "rmsnorm": lambda: nm.nm_rmsnorm_mx4(x, None, r, q=q, scales=s, residual_out=out),
            "dequantize": lambda: nm.nm_dequantize_mx4(q, s, y=out),
            "pack": lambda: nm.nm_mx4_pack(Tensor((64, 32), u8, dev), Tensor((64, 2), u8, dev)),
            "linear": lambda: nm.nm_linear_mx4(q, s, packed, y=out),
            "linear rounded": lambda: nm.nm_linear_mx4(q, s, packed, y=yq, y_scales=ys, rounded=True),
            "experts": lambda: nm.nm_experts_mx4(q, s, several, offsets, rows, y=out),
            "route": lambda: nm.nm_route(Made((3, 8), f32, dev), 2),
            "combine": lambda: nm.nm_combine(x, Tensor((3, 2), i32, dev), Tensor((3, 2), f32, dev), r, out=out)}


@pytest.mark.parametrize("name", sorted(_calls(0)))
def test_tensors_of_another_device_are_refused(machine, name):  # noqa: F811
    with pytest.raises(ValueError, match="device 1"):
        _calls(1)[name]()
    assert machine.launches == 0
    _calls(0)[name]()
    assert machine.launches == 1


@pytest.mark.parametrize("name", ["scales", "offsets", "rows", "y", "bias"])
def test_one_tensor_of_another_device_is_refused(machine, name):  # noqa: F811
    def at(which):
        return 1 if which == name else 0
    i32, u8 = torch.int32, torch.uint8
    with pytest.raises(ValueError, match="device 0"):
        nm.nm_experts_mx4(Tensor((3, 32), u8, 0), Tensor((3, 2), u8, at("scales")), nm.MX4Weights(None, 2, 64, 64, False), Tensor((3,), i32, at("offsets")),
                          Tensor((3,), i32, at("rows")), Tensor((2, 64), torch.float32, at("bias")), y=Tensor((3, 64), torch.float32, at("y")))
    assert machine.launches == 0


def _weights(experts, channels, width, gated):
    return nm.MX4Weights(None, experts, channels, width, gated)


@pytest.mark.parametrize("x,logits", [((5, 64), (4, 3)), ((4, 64), (5, 3)), ((2, 2, 64), (4, 3)), ((4, 64), (4, 2)), ((4, 64), (4, 4))])
def test_rows_and_logits_that_do_not_fit_together_are_refused(machine, x, logits):  # noqa: F811
    layer = ExpertsMX4(_weights(3, 128, 64, True), _weights(3, 64, 64, False), 2)
    with pytest.raises(ValueError, match="do not fit together"):
        layer(Tensor(x, torch.float32, 0), Tensor(logits, torch.float32, 0))
    assert machine.launches == 0


def test_weights_that_do_not_fit_together_are_refused():
    up, down = _weights(3, 128, 64, True), _weights(3, 64, 64, False)
    for a, b, k in ((down, down, 2), (up, up, 2), (up, _weights(3, 64, 96, False), 2), (up, _weights(3, 96, 64, False), 2), (up, _weights(2, 64, 64, False), 2), (up, down, 0),
                    (up, down, 4)):
        with pytest.raises(ValueError):
            ExpertsMX4(a, b, k)
    with pytest.raises(ValueError):
        FeedForwardMX4(None, up, down)
