"""A product in MX4 of more workgroups than one launch has room for."""
import pytest
import torch

from paper_2507_17301_amd import binding as nm
from gpu_util import say
from mx4_util import random_mx4

pytestmark = pytest.mark.gpu


def test_products_of_several_launches():
    """2^24 workgroups of 256 threads are the first that do not fit; outputs of 18 GB."""
    rows, k, n = (1 << 22) + 77, 64, 1 << 14
    g = torch.Generator().manual_seed(4)
    h = nm.nm_mx4_pack(*(v.cuda() for v in random_mx4(g, (n, k), 110, 122)), k, gated=True)
    q, s = (v.cuda() for v in random_mx4(g, (rows, k)))
    say(f"linear_mx4 {rows} x {k} x {n} gated, MX4")
    y, ys = torch.zeros((rows, n // 4), dtype=torch.uint8, device="cuda"), torch.zeros((rows, n // 64), dtype=torch.uint8, device="cuda")
    nm.nm_linear_mx4(q, s, h, y=y, y_scales=ys, rounded=True)
    part = 1 << 19
    for at in range(0, rows, part):
        a, b = nm.nm_linear_mx4(q[at:at + part], s[at:at + part], h, rounded=True)
        assert torch.equal(y[at:at + part], a) and torch.equal(ys[at:at + part], b), at
    assert (ys[-77:] > 0).all()
    del y, ys
    torch.cuda.empty_cache()
