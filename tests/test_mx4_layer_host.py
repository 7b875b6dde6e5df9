"""What the layer of experts refuses before anything is launched, with stand-ins for the tensors and the library: no GPU is needed."""
import pytest
import torch

from paper_2507_17301_amd.feedforward import ExpertsMX4
from test_mx4_device import Made, _weights
from test_q8_device import machine, pytestmark  # noqa: F401  (the fixture and the mark)


def test_types_of_the_answers():
    up, down = _weights(3, 128, 64, True), _weights(3, 64, 64, False)
    assert ExpertsMX4(up, down, 2).answers == torch.float32 and ExpertsMX4(up, down, 2, answers=torch.bfloat16).answers == torch.bfloat16
    for bad in (torch.float16, torch.int32):
        with pytest.raises(ValueError, match="fp32 or bf16"):
            ExpertsMX4(up, down, 2, answers=bad)


@pytest.mark.parametrize("width", [1, 32, 33, 63, 65, 96])
def test_rows_of_another_width_are_refused(machine, width):  # noqa: F811
    """Of 33 to 63 values, too, which have as many blocks as the weights' 64."""
    layer = ExpertsMX4(_weights(3, 128, 64, True), _weights(3, 64, 64, False), 2)
    with pytest.raises(ValueError, match=f"rows of {width} values"):
        layer(Made((4, width), torch.float32, 0), Made((4, 3), torch.float32, 0))
    assert machine.launches == 0
