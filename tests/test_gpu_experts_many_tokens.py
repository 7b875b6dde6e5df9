"""Routing of more tokens than 256 batches of 64, whose counts are whole numbers of 32 bits, over few and many experts."""
import math

import pytest
import torch

from paper_2507_17301_amd import binding as nm
from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,experts,k", [(16385, 1024, 3), (20000, 300, 8), (33000, 65, 2), (70001, 1, 1), (40000, 256, 8)])
def test_many_tokens(tokens, experts, k, dtype):
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, experts), generator=g)
    x = ((x * 4).round() / 4 if experts % 2 else x).to(dtype)             # (many ties)
    x[::11] = -math.inf                                                   # padding
    say(f"route {tokens} x {experts} k {k} {dtype}")
    got = nm.nm_route(x.cuda(), k)
    best, ids = torch.sort(x.float(), dim=1, descending=True, stable=True)
    ids = torch.where(best[:, :k] == -math.inf, -1, ids[:, :k])
    assert torch.equal(got.ids.cpu().long(), ids)
    flat = torch.where(ids < 0, experts, ids).flatten()
    by, order = torch.sort(flat, stable=True)
    end = int((flat < experts).sum())
    counts = torch.bincount(flat, minlength=experts + 1)[:experts]
    assert got.offsets.tolist() == [0] + counts.cumsum(0).tolist()
    assert torch.equal(got.rows.cpu().long(), torch.where(torch.arange(tokens * k) < end, order // k, -1))
    slots = torch.empty_like(order)
    slots[order] = torch.arange(tokens * k)
    assert torch.equal(got.slots.cpu().long(), torch.where(ids < 0, -1, slots.view(tokens, k)))
    weights = torch.softmax(torch.where(ids < 0, -math.inf, best[:, :k].double()), dim=1).nan_to_num(0.0)
    # exp's own 2 u and its argument's rounding, k terms, the quotient
    assert (got.weights.cpu().double() - weights).abs().max() <= (2 * 2 * 8 + 8 + k) * 2.0 ** -24
