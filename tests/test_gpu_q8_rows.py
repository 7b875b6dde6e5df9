"""The row operators in 8 bits (norm, rounding, reading back) against their formulas in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2507_17301_amd import binding as nm
from gpu_util import say
from q8_util import U, check_rounded, on_gpu, rows_of

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# one group of 8 and its neighbours, every thread arrangement's ends, odd widths, the longest row
WIDTHS = [1, 2, 7, 8, 9, 63, 64, 511, 512, 513, 1000, 1024, 1025, 2048, 2051, 4096, 4099, 8192, 8195, 16384, 16391, 32768, 32775, 65536]


def _rows(width):
    return 1 if width > 30000 else 5


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("width", WIDTHS)
def test_rounding_and_reading_back(width, dtype):
    g = torch.Generator().manual_seed(width)
    x = rows_of(g, _rows(width), width, TYPES[dtype])
    say(f"quantize {tuple(x.shape)} {dtype}")
    q, s = nm.nm_quantize_q8(x.cuda())
    torch.cuda.synchronize()
    x64 = x.double().numpy()
    check_rounded(q, s, x64, 0.0)
    assert np.array_equal(s.cpu().numpy(), (np.abs(x.float().numpy()).max(axis=1) / np.float32(127)).astype(np.float32))
    for out in (torch.float32, torch.bfloat16):
        y = nm.nm_dequantize_q8(q, s, out)
        assert torch.equal(y, (q.float() * s[:, None]).to(out))


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("width", WIDTHS)
def test_norm(width, residual, dtype):
    g = torch.Generator().manual_seed(width + 1)
    x = rows_of(g, _rows(width), width, TYPES[dtype])
    r = rows_of(g, _rows(width), width, TYPES[dtype]) if residual else None
    gamma = 1 + 0.2 * torch.randn(width, generator=g)
    eps = 1e-5
    say(f"norm {tuple(x.shape)} {dtype} residual {residual}")
    q, s, h = nm.nm_rmsnorm_q8(x.cuda(), gamma.cuda(), r.cuda() if residual else None, eps)
    torch.cuda.synchronize()
    h32 = x.float() + r.float() if residual else x.float()
    if residual:
        assert torch.equal(h.cpu(), h32.to(x.dtype))
    else:
        assert h is None
    h64 = h32.double().numpy()      # (the sum of two bf16 or fp32 values is formed in fp32, with one rounding)
    v = gamma.double().numpy() * h64 / np.sqrt((h64 ** 2).mean(axis=1, keepdims=True) + eps)
    check_rounded(q, s, v, 1e-5)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,width,gap", [(3, 40, 1), (9, 1001, 3), (300, 520, 8), (130, 2051, 5), (1, 77, 9)])
def test_strided_rows_are_the_same(rows, width, gap, dtype):
    g = torch.Generator().manual_seed(rows)
    x, r = rows_of(g, rows, width, TYPES[dtype], gap), rows_of(g, rows, width, TYPES[dtype], gap + 2)
    xd, rd = on_gpu(x, width), on_gpu(r, width)
    say(f"strided norm {rows} x {width} + {gap} {dtype}")
    q, s, h = nm.nm_rmsnorm_q8(xd.contiguous(), None, rd.contiguous())
    qw, hw = torch.full((rows, width + 3), 99, dtype=torch.int8, device="cuda"), torch.full((rows, width + 1), 7.0, dtype=x.dtype, device="cuda")
    q2, s2, h2 = nm.nm_rmsnorm_q8(xd, None, rd, q=qw[:, 2:2 + width], residual_out=hw[:, 1:])
    assert torch.equal(q, q2) and torch.equal(s, s2) and torch.equal(h, h2)
    assert (qw[:, :2] == 99).all() and (qw[:, 2 + width:] == 99).all() and (hw[:, 0] == 7).all()
    yw = torch.full((rows, width + 5), 3.0, device="cuda")
    nm.nm_dequantize_q8(q2, s2, y=yw[:, 4:4 + width])
    assert torch.equal(yw[:, 4:4 + width], q.float() * s[:, None]) and (yw[:, :4] == 3).all() and (yw[:, 4 + width:] == 3).all()
    # columns of one wide tensor, read and written in one call; a row repeated by stride 0; the stream updated in place
    wide = torch.cat([xd, rd], 1).contiguous()
    q3, s3, _ = nm.nm_rmsnorm_q8(wide[:, :width], None, rd, residual_out=wide[:, width:])
    assert torch.equal(q3, q) and torch.equal(s3, s) and torch.equal(wide[:, width:], h)
    same = xd[:1].expand(rows, width)
    q4, s4 = nm.nm_quantize_q8(same)
    q5, s5 = nm.nm_quantize_q8(xd[:1].contiguous())
    assert torch.equal(q4, q5.expand(rows, width)) and torch.equal(s4, s5.expand(rows))
    for base in ("x", "residual"):
        xc, rc = xd.contiguous().clone(), rd.contiguous().clone()
        out = xc if base == "x" else rc
        q6, s6, h6 = nm.nm_rmsnorm_q8(xc, None, rc, residual_out=out)
        assert h6 is out and torch.equal(out, h) and torch.equal(q6, q) and torch.equal(s6, s)


@pytest.mark.parametrize("width", [5, 64, 700, 1500, 4096, 20000])
def test_rows_that_are_zero_tiny_or_not_finite(width):
    g = torch.Generator().manual_seed(width)
    x = torch.randn((9, width), generator=g)
    x[1] = 0
    x[2, width // 2] = math.nan
    x[3, width - 1] = math.inf
    x[4, 0] = -math.inf
    x[5] *= 1e-38                 # below what counts as zero
    x[6] *= 1e-15 / x[6].abs().max()
    x[7] *= 3e38 / x[7].abs().max()   # squares overflow fp32
    say(f"special rows of {width}")
    for norm in (False, True):
        q, s = nm.nm_rmsnorm_q8(x.cuda(), None, None, 0.0)[:2] if norm else nm.nm_quantize_q8(x.cuda())
        y = nm.nm_dequantize_q8(q, s).cpu()
        # without eps, 0 / 0, squares that underflow to it and squares past fp32 are not finite either
        bad, zero = ((1, 2, 3, 4, 5, 7), ()) if norm else ((2, 3, 4), (1, 5))
        for i in range(9):
            if i in bad:
                assert torch.isnan(s[i]) and not q[i].any() and torch.isnan(y[i]).all()
            elif i in zero:
                assert s[i] == 0 and not q[i].any() and not y[i].any()
            else:
                v = x[i].double().numpy()[None]
                check_rounded(q[i:i + 1], s[i:i + 1], v / np.sqrt((v ** 2).mean()) if norm else v, 1e-5 if norm else 0.0)
    q, s, _ = nm.nm_rmsnorm_q8(x.cuda(), None, None, 1e-6)
    assert s[1] == 0 and not q[1].any()
    # a gain that is not finite spoils every row that it touches, whatever its value there
    gamma = torch.ones(width)
    gamma[width // 3] = math.nan
    q, s, _ = nm.nm_rmsnorm_q8(x.cuda(), gamma.cuda())
    assert torch.isnan(s).all() and not q.any()


def test_no_rows_more_axes_and_many_rows():
    e = torch.empty((0, 64), device="cuda")
    q, s = nm.nm_quantize_q8(e)
    assert q.shape == (0, 64) and s.shape == (0,) and nm.nm_dequantize_q8(q, s).shape == (0, 64)
    x = torch.randn((2, 3, 50), device="cuda")
    q, s, h = nm.nm_rmsnorm_q8(x, None, x)
    q2, s2, h2 = nm.nm_rmsnorm_q8(x.view(6, 50), None, x.view(6, 50))
    assert q.shape == (2, 3, 50) and s.shape == (2, 3) and torch.equal(q.view(6, 50), q2) and torch.equal(h.view(6, 50), h2)
    one = torch.randn(50, device="cuda")
    assert nm.nm_quantize_q8(one)[1].shape == ()
    # more rows than a launch has workgroups
    rows = (1 << 20) * 4 + 3
    x = torch.randn((rows, 2), device="cuda")
    q, s = nm.nm_quantize_q8(x)
    assert np.array_equal(s.cpu().numpy(), np.abs(x.cpu().numpy()).max(axis=1) / np.float32(127))
    assert torch.equal(nm.nm_dequantize_q8(q, s), q.float() * s[:, None])


@pytest.mark.parametrize("norm", [False, True])
def test_workgroups_that_take_several_rows(norm):
    """More rows than workgroups, and rows that a workgroup's wavefronts share: one row's reductions do not meet the next one's."""
    rows, width = (1 << 20) + 5000, 1032
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((4096, width), generator=g, device="cuda").to(torch.bfloat16)
    x *= torch.exp(torch.randn(4096, generator=g, device="cuda") * 3)[:, None].to(torch.bfloat16)
    many = x.repeat(rows // 4096 + 1, 1)[:rows]
    say(f"{rows} rows of {width}, norm {norm}")
    call = (lambda t: nm.nm_rmsnorm_q8(t)[:2]) if norm else nm.nm_quantize_q8
    q0, s0 = call(x)
    q, s = call(many)
    for i in range(0, rows, 4096):
        n = min(4096, rows - i)
        assert torch.equal(q[i:i + n], q0[:n]) and torch.equal(s[i:i + n], s0[:n])


def test_offsets_past_32_bits():
    """Rows whose bytes lie more than 4 GiB apart."""
    rows, width, ld = 3, 1000, 1 << 24
    wide = torch.empty((65 * ld + width,), dtype=torch.float32, device="cuda")      # 4.4 GB
    x = wide.as_strided((66, width), (ld, 1))
    x.copy_(torch.randn((66, width), device="cuda"))
    say("rows 64 MiB apart, over 4 GiB")
    q, s = nm.nm_quantize_q8(x)
    qc, sc = nm.nm_quantize_q8(x.contiguous())
    assert torch.equal(q, qc) and torch.equal(s, sc)


def test_the_current_stream_and_a_given_one():
    x = torch.randn((64, 4096), device="cuda", dtype=torch.bfloat16)
    q0, s0 = nm.nm_quantize_q8(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x2 = x * 2
        q, s = nm.nm_quantize_q8(x2)
    q1, s1 = torch.empty_like(q0), torch.empty_like(s0)
    nm.nm_quantize_q8(x2, q1, s1, stream=side)
    side.synchronize()
    assert torch.equal(q, q0) and torch.equal(s, s0 * 2) and torch.equal(q1, q0) and torch.equal(s1, s)


def test_refusals():
    x = torch.randn((4, 64), device="cuda")
    with pytest.raises(ValueError):
        nm.nm_quantize_q8(x.cpu())
    with pytest.raises(ValueError):
        nm.nm_quantize_q8(x.t())                      # a row's values are not adjacent
    with pytest.raises(ValueError):
        nm.nm_rmsnorm_q8(x, torch.ones(63, device="cuda"))
    with pytest.raises(ValueError):
        nm.nm_rmsnorm_q8(x, None, x[:2])
    with pytest.raises(TypeError):
        nm.nm_quantize_q8(x.half())
    with pytest.raises(TypeError):
        nm.nm_dequantize_q8(x, x[:, 0].contiguous())
    for eps in (-1.0, math.nan, math.inf):
        with pytest.raises(nm.NMError) as e:
            nm.nm_rmsnorm_q8(x, eps=eps)
        assert e.value.code == nm.NM_ERR_ARG
    with pytest.raises(nm.NMError) as e:
        nm.nm_quantize_q8(torch.zeros((1, nm.NM_Q8_MAX_WIDTH + 1), device="cuda"))
    assert e.value.code == nm.NM_ERR_SHAPE
    with pytest.raises(nm.NMError) as e:
        nm.nm_quantize_q8(torch.zeros((2, 0), device="cuda"))
    assert e.value.code == nm.NM_ERR_ARG
    wide = torch.randn((4, 100), device="cuda")
    with pytest.raises(nm.NMError) as e:               # the stream may be x itself, not x moved by some columns
        nm.nm_rmsnorm_q8(wide[:, :64], None, x, residual_out=wide[:, 1:65])
    assert e.value.code == nm.NM_ERR_ARG and "overlaps" in str(e.value)
    out = torch.empty((1, 64), dtype=torch.int8, device="cuda").expand(4, 64)
    with pytest.raises(nm.NMError) as e:               # rows of an output lie apart
        nm.nm_quantize_q8(x, q=out)
    assert e.value.code == nm.NM_ERR_ARG
