"""Every kernel that a product in 8 bits can take, at sizes where each is chosen: wide layers with few rows, tiles of all shapes,
sums divided over workgroups, outputs stored past the cache, offsets beyond 32 bits.  References in 64 bits, on the GPU."""
import pytest
import torch

from paper_2507_17301_amd import binding as nm
from gpu_util import say
from q8_util import U

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _inputs(rows, k, n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(-127, 128, (rows, k), generator=g, dtype=torch.int8, device="cuda")
    w = torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8, device="cuda")
    s = (0.5 + torch.rand(rows, generator=g, device="cuda")) / 100
    ws = (0.5 + torch.rand(n, generator=g, device="cuda")) / (70 * k ** 0.5)
    return q, s, w, ws, torch.randn(n, generator=g, device="cuda")


def _check(y, q, s, w, ws, bias, residual, gated, step=1024):
    """As q8_util.linear_ref and check_close, a part of the rows at a time."""
    wt = w.double().t().contiguous()
    for i in range(0, y.shape[0], step):
        a = (q[i:i + step].double() @ wt) * s[i:i + step, None].double() * ws.double()
        z, e = a, 4 * U * a.abs()
        if bias is not None:
            z, e = a + bias.double(), e + 4 * U * bias.double().abs()
        if gated:
            half = z.shape[1] // 2
            g, v = z[:, :half], z[:, half:]
            ref = g * torch.sigmoid(g) * v
            bound = 1.1 * e[:, :half] * v.abs() + (g * torch.sigmoid(g)).abs() * e[:, half:] + ref.abs() * (2 * g.abs() + 8) * U + 1e-37
        elif residual is not None:
            r = residual[i:i + step].double()
            ref, bound = z + r, e + 2 * U * (z.abs() + r.abs())
        else:
            ref, bound = z, e
        if y.dtype == torch.bfloat16:
            bound = bound + 2.0 ** -8 * (ref.abs() + bound) + 2.0 ** -133
        got = y[i:i + step].double()
        assert torch.isfinite(got).all()
        assert ((got - ref).abs() <= bound).all(), ((got - ref).abs() - bound).max()


def _product(rows, k, n, dtype, gated=False, bias=True, residual=False, seed=1):
    q, s, w, ws, b = _inputs(rows, k, n, seed)
    say(f"product {rows} x {k} x {n} {dtype} gated {gated} bias {bias} residual {residual}")
    h = nm.nm_q8_pack(w, ws, gated=gated)
    r = torch.randn((rows, n), device="cuda").to(TYPES[dtype]) if residual else None
    y = nm.nm_linear_q8(q, s, h, b if bias else None, r, TYPES[dtype])
    torch.cuda.synchronize()
    _check(y, q, s, w, ws, b if bias else None, r, gated)


# channels at which a workgroup of the few-row kernels takes one, two or four blocks of 16
@pytest.mark.parametrize("n", [8128, 8200, 12224, 12290])
@pytest.mark.parametrize("rows", [1, 9, 16, 17, 32, 33, 50, 64])
def test_few_rows_on_many_channels(rows, n):
    for k, gated, dtype in ((64, False, "bf16"), (200, True, "bf16"), (1000, False, "f32")):
        _product(rows, k, n, dtype, gated, residual=not gated and rows % 2 == 1, seed=rows)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,k,n", [(65, 4096, 1000), (100, 12288, 300), (128, 2048, 520), (300, 4096, 4096), (300, 1200, 9000),
                                      (700, 8192, 200), (1000, 4096, 4100), (1500, 16000, 300), (2049, 272, 5003), (4100, 512, 4400)])
def test_tiles_and_divided_sums(rows, k, n, dtype, residual):
    _product(rows, k, n, dtype, False, True, residual, seed=rows)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,k,n", [(65, 4096, 1000), (130, 8192, 514), (300, 4096, 8192), (1000, 1030, 6002), (2600, 256, 10000)])
def test_gated_tiles_and_divided_sums(rows, k, n, dtype):
    _product(rows, k, n, dtype, True, True, seed=rows)


# 256 channels x 256, 192, 128 rows, 128 channels x 192, 160, 128, 64; each whole and divided
@pytest.mark.parametrize("form", ["plain", "residual", "gated"])
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,k,n", [(2696, 68, 4618), (12517, 14626, 148), (4741, 66, 1734), (8213, 12060, 134), (3273, 67, 1794),
                                      (850, 7280, 2796), (979, 64, 5286), (165, 5056, 4684), (150, 1005, 10058), (131, 3427, 1618),
                                      (83, 215, 68), (84, 3864, 1172), (91, 260, 78), (67, 2615, 96)])
def test_each_shape_of_tile(rows, k, n, dtype, form):
    _product(rows, k, n, dtype, form == "gated", True, form == "residual", seed=k)


@pytest.mark.parametrize("rows,n,dtype,gated,residual", [(5000, 17000, "bf16", False, False), (5000, 17001, "bf16", False, True),
                                                         (3000, 14003, "f32", False, False), (6000, 30002, "bf16", True, False)])
def test_outputs_stored_past_the_cache(rows, n, dtype, gated, residual):
    _product(rows, 80, n, dtype, gated, True, residual, seed=3)


def test_the_same_bits_with_and_without_a_workspace_path():
    """Unaligned rows are copied first, divided sums are joined: neither shows in the result."""
    for rows, k, n in ((20, 4000, 520), (100, 4000, 520), (333, 1040, 2501)):
        q, s, w, ws, b = _inputs(rows, k, n, rows)
        h = nm.nm_q8_pack(w, ws)
        whole = nm.nm_linear_q8(q, s, h, b, dtype=torch.float32)
        odd = torch.zeros((rows, k + 3), dtype=torch.int8, device="cuda")[:, 3:]
        odd.copy_(q)
        assert torch.equal(nm.nm_linear_q8(odd, s, h, b, dtype=torch.float32), whole)
        assert torch.equal(nm.nm_linear_q8(q[:1], s[:1], h, b, dtype=torch.float32), whole[:1])


def test_workspace_paths_in_a_graph():
    q, s, w, ws, b = _inputs(100, 4000, 520, 8)
    h = nm.nm_q8_pack(w, ws)
    odd = torch.zeros((100, 4003), dtype=torch.int8, device="cuda")[:, 3:]
    inputs = [torch.randint(-127, 128, (100, 4000), dtype=torch.int8, device="cuda") for _ in range(3)]
    want = [nm.nm_linear_q8(x, s, h, b) for x in inputs]
    odd.copy_(inputs[0])
    nm.nm_linear_q8(odd, s, h, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = nm.nm_linear_q8(odd, s, h, b)
    for i in (1, 0, 2, 1):
        odd.copy_(inputs[i])
        graph.replay()
        assert torch.equal(y, want[i])
        _ = y.float().sum().item()


def test_offsets_past_32_bits():
    """Rows of q, of the residual and of the output 16 million elements apart."""
    rows, k, n, ld = 300, 96, 70, 1 << 24
    q, s, w, ws, b = _inputs(rows, k, n, 5)
    h = nm.nm_q8_pack(w, ws)
    say("strides of 2^24 elements, offsets over 10 GB")
    wide = torch.empty((rows - 1) * ld + 256, dtype=torch.bfloat16, device="cuda")
    y, r = wide.as_strided((rows, n), (ld, 1)), wide.as_strided((rows, n), (ld, 1), 100)
    r.copy_(torch.randn((rows, n), device="cuda"))
    qw = torch.empty((rows - 1) * ld + k, dtype=torch.int8, device="cuda").as_strided((rows, k), (ld, 1))
    qw.copy_(q)
    nm.nm_linear_q8(qw, s, h, b, residual=r, y=y)
    assert torch.equal(y, nm.nm_linear_q8(q, s, h, b, residual=r.contiguous()))
    nm.nm_linear_q8(qw[:40], s[:40], h, b, residual=r[:40], y=y[:40])
    assert torch.equal(y[:40], nm.nm_linear_q8(q[:40], s[:40], h, b, residual=r[:40].contiguous()))


def test_a_freed_handle_is_refused():
    q, s, w, ws, _ = _inputs(4, 64, 32, 1)
    h = nm.nm_q8_pack(w, ws)
    h.free()
    for rows in (1, 4):
        with pytest.raises(nm.NMError) as e:
            nm.nm_linear_q8(q[:rows], s[:rows], h)
        assert e.value.code == nm.NM_ERR_ARG
