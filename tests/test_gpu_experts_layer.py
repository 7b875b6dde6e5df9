"""The layer of experts against its formula in 64 bits, where a rounding of the experts' answers would show."""

import pytest
import torch

from paper_2507_17301_amd import binding as nm
from paper_2507_17301_amd.feedforward import ExpertsMX4
from gpu_util import say
from mx4_util import U, check_close, random_mx4, rows_of, values_of
from test_gpu_experts import TYPES, grouped_ref, route_ref

pytestmark = pytest.mark.gpu


def weights_of(g, experts, width, hidden):
    """Codes and scales of the gated and of the second products' weights."""
    return random_mx4(g, (experts, 2 * hidden, width), 116, 122), random_mx4(g, (experts, width, hidden), 116, 122)


@pytest.mark.parametrize("answers", [None, torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("tokens,k", [(1, 1), (40, 1), (40, 3), (700, 4)])
def test_answers_are_rounded_as_asked(tokens, k, dtype, answers):
    """A residual that takes back the rounded sum leaves what the roundings before it did."""
    dtype = TYPES[dtype]
    g = torch.Generator().manual_seed(tokens + k)
    experts, width, hidden = 7, 192, 160
    (w1, s1), (w2, s2) = weights_of(g, experts, width, hidden)
    up, down = nm.nm_mx4_pack(w1.cuda(), s1.cuda(), width, gated=True), nm.nm_mx4_pack(w2.cuda(), s2.cuda(), hidden)
    layer = ExpertsMX4(up, down, k) if answers is None else ExpertsMX4(up, down, k, answers=answers)
    x, logits = rows_of(g, tokens, width, dtype).cuda(), torch.randn((tokens, experts), generator=g)
    say(f"ExpertsMX4 {tokens} tokens, {k} choices, {dtype}, answers {answers}")
    _, weights, offsets, rows, slots = route_ref(logits, k)
    to = nm.nm_route(logits.cuda(), k)
    # what the second product gets is the kernel's own rounding
    q, s = nm.nm_experts_mx4(*nm.nm_quantize_mx4(x), up, to.offsets, to.rows, rounded=True)
    y, bound = grouped_ref(values_of(q, s, hidden), offsets, values_of(w2, s2, hidden), None, False)
    if answers == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (y.abs() + bound)
    terms = weights[..., None] * y[slots]
    r = (-terms.sum(dim=1)).to(dtype)
    ref = terms.sum(dim=1) + r.double()
    # the weights: (2 * spread + 8 + experts) u as for the routing; each of the k products and sums, the residual's sum: a rounding
    spread = 2 * float(logits.abs().max())
    size = terms.abs().sum(dim=1) + r.double().abs()
    err = (weights[..., None] * bound[slots]).sum(dim=1) + (2 * spread + 8 + experts + k + 2) * U * size
    out = layer(x, logits.cuda(), r.cuda())
    assert out.dtype == dtype
    check_close(out, ref, err)
    if answers is None:
        assert torch.equal(out, ExpertsMX4(up, down, k, answers=torch.float32)(x, logits.cuda(), r.cuda()))
