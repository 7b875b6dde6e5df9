"""What the layer of experts refuses before anything is launched, with stand-ins for the tensors and the library: no GPU is needed."""
import pytest
import torch

from paper_2507_17301_amd.feedforward import ExpertsMX4
from test_mx4_device import _weights
from test_q8_device import pytestmark  # noqa: F401  (the mark)


def test_types_of_the_answers():
    up, down = _weights(3, 128, 64, True), _weights(3, 64, 64, False)
    assert ExpertsMX4(up, down, 2).answers == torch.float32 and ExpertsMX4(up, down, 2, answers=torch.bfloat16).answers == torch.bfloat16
    for bad in (torch.float16, torch.int32):
        with pytest.raises(ValueError, match="fp32 or bf16"):
            ExpertsMX4(up, down, 2, answers=bad)
