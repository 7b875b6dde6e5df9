"""The gated products' silu over the range of its gates.  Weights of zero leave the bias, so that gate and value are exactly known.

silu4's bound, with u = 2^-24: (2 |gate| + 12) u of the result (the exponential's argument and the instruction, both counted twice, the
reciprocal, one rounding for the sum and each of four products), and the last subnormal digit; one rounding more to bf16."""
import pytest
import torch

from paper_2507_17301_amd import binding as nm
from gpu_util import say
from mx4_util import U, blocks, check_close, check_rounded

pytestmark = pytest.mark.gpu

# gates and what they are multiplied with: results within fp32's range
RANGES = {"around -88": (-89.0, -86.0, 1e30), "from -174": (-174.0, -80.0, 3e37), "negative": (-90.0, -1e-3, -2.0), "around 0": (-1.0, 1.0, 1e-3),
          "positive": (1e-3, 200.0, 1e30), "large": (1e3, 1e30, -1e7)}


# few rows, one matrix's tiles of 64 and of 128 rows
@pytest.mark.parametrize("rows", [3, 40, 600, 2500])
@pytest.mark.parametrize("name", sorted(RANGES))
def test_silu(name, rows):
    low, high, up = RANGES[name]
    n, k = 1440, 128
    gate = torch.linspace(low, high, n, dtype=torch.float64).float()
    value = (up * (1.0 + torch.arange(n) % 7 / 8.0)).float()
    h = nm.nm_mx4_pack(torch.zeros((2 * n, k), device="cuda"), gated=True)
    q, s = torch.zeros((rows, 64), dtype=torch.uint8, device="cuda"), torch.full((rows, blocks(k)), 127, dtype=torch.uint8, device="cuda")
    g, v = gate.double(), value.double()
    ref = g / (1.0 + torch.exp(-g)) * v
    bound = (2 * g.abs() + 12) * U * ref.abs() if name != "large" else 12 * U * ref.abs()   # (s is 0 there)
    bound = bound + 2.0 ** -148
    ref, bound = ref.expand(rows, n), bound.expand(rows, n)
    say(f"silu {name}, {rows} rows")
    bias = torch.cat([gate, value]).cuda()
    check_close(nm.nm_linear_mx4(q, s, h, bias, dtype=torch.float32), ref, bound)
    check_close(nm.nm_linear_mx4(q, s, h, bias), ref, bound)
    check_rounded(*nm.nm_linear_mx4(q, s, h, bias, rounded=True), ref, bound)


@pytest.mark.parametrize("rows", [3, 2500])
def test_gates_past_the_range(rows):
    """Under -174 the result is 0; infinities and NaN as in the formula."""
    n, k = 1440, 128
    gate, value = torch.full((n,), -175.0), torch.full((n,), 1e30)
    gate[1], gate[2], gate[3], gate[4], gate[5] = -1e30, float("inf"), -float("inf"), float("nan"), 0.0
    value[6] = float("nan")
    h = nm.nm_mx4_pack(torch.zeros((2 * n, k), device="cuda"), gated=True)
    q, s = torch.zeros((rows, 64), dtype=torch.uint8, device="cuda"), torch.full((rows, blocks(k)), 127, dtype=torch.uint8, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        y = nm.nm_linear_mx4(q, s, h, torch.cat([gate, value]).cuda(), dtype=dtype).float().cpu()
        assert (y[:, 2] == float("inf")).all() and torch.isnan(y[:, [3, 4, 6]]).all()
        rest = [i for i in range(n) if i not in (2, 3, 4, 6)]
        assert (y[:, rest] == 0).all()
