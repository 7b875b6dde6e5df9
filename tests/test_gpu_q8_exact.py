"""Where the 8-bit operators have one right answer, or an error bound that the magnitudes of the values do not widen."""
import numpy as np
import pytest
import torch

from paper_2507_17301_amd import binding as nm
from gpu_util import say

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _every_pair():
    """Rows that hold every bf16 significand at every binade that does not round to 0, of both signs, under every largest magnitude:
    (values fp32 [128, n], x * 127 / a rounded to the nearest, ties to even, in whole numbers [128, n])."""
    m, j = np.meshgrid(np.arange(128, 256), np.arange(10), indexing="ij")
    m, j = m.reshape(-1), j.reshape(-1)                      # a value is m * 2^-j
    rows, want = [], []
    for a in range(128, 256):
        there = (m <= (a << j)) & ~((j == 0) & (m > a))
        num, den = 127 * m, a << j
        q = num // den
        twice = 2 * (num - q * den)
        q = q + ((twice > den) | ((twice == den) & (q % 2 == 1)))
        value, q = np.where(there, m * 2.0 ** -j, 0.0), np.where(there, q, 0)
        rows.append(np.concatenate([value, -value, [a]]))
        want.append(np.concatenate([q, -q, [127]]))
    return torch.from_numpy(np.array(rows, dtype=np.float32)), torch.from_numpy(np.array(want, dtype=np.int8))


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_rounding_of_bf16_values_is_to_the_nearest_ties_to_even(dtype):
    """a = 3, x = 1.5 is 63.5 and gives 64, although 127 / 3 is no fp32 number."""
    x, want = _every_pair()
    for power in (0, -100, 100):
        xs = (x * 2.0 ** power).to(TYPES[dtype])
        assert torch.equal(xs.double(), x.double() * 2.0 ** power)
        say(f"every pair of bf16 significands x 2^{power} as {dtype}")
        q, _ = nm.nm_quantize_q8(xs.cuda())
        off = (q.cpu() != want)
        assert not off.any(), f"{int(off.sum())} of {off.numel()}, first {xs[off][0]} in row {int(off.nonzero()[0, 0])}: {q.cpu()[off][0]} for {want[off][0]}"
        # channels of weights are rounded the same way
        assert np.array_equal(nm.nm_q8_export(nm.nm_q8_pack(xs.cuda()))[0], want.numpy())
