"""Products in 8 bits whose K is long against the stages in LDS: stages are loaded again and again in each other's place, with the waits of
the middle of the loop, whole and partial last steps.  References in 64 bits."""
import pytest

from q8_cases import FEW_CHANNELS, FEW_ROWS, FEW_WIDTHS, RING
from test_gpu_q8_paths import TYPES, _product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", ["plain", "residual", "gated"])
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("shape", sorted(RING))
def test_undivided_tiles(shape, dtype, form):
    for rows, k, n in RING[shape]:
        _product(rows, k, n, dtype, form == "gated", True, form == "residual", seed=rows)


@pytest.mark.parametrize("form", ["plain", "residual", "gated"])
@pytest.mark.parametrize("n", FEW_CHANNELS)
@pytest.mark.parametrize("k", FEW_WIDTHS)
def test_few_rows(k, n, form):
    for i, rows in enumerate(FEW_ROWS):
        _product(rows, k, n, "f32" if i % 2 else "bf16", form == "gated", True, form == "residual", seed=rows + k)
