"""Rounding to MX4, its norm and its reading back against their formulas in 64 bits: codes and scales are those, exactly."""
import math

import pytest
import torch

from paper_2507_17301_amd import binding as nm
from gpu_util import say
from mx4_util import blocks, on_gpu, random_mx4, round_ref, rows_of, same, values_of

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# one, odd ones, the ends of blocks, and of each number of threads that a norm's row is dealt to
WIDTHS = [1, 2, 31, 32, 33, 63, 100, 257, 512, 513, 1000, 1024, 1030, 2048, 2050, 4096, 5001, 6150, 8192, 8200, 16384, 20000, 40000, 65536]


def norm_ref(x, r, gamma, eps):
    """v of the norm: single operations in fp32 but for n, a 64-bit number rounded once; and h."""
    h = x.float() if r is None else x.float() + r.float()
    n = (1.0 / torch.sqrt((h.double() ** 2).mean(dim=1, keepdim=True) + eps)).float()
    v = h * n
    return (v if gamma is None else v * gamma), h


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("width", WIDTHS)
def test_rounding(width, dtype):
    for rows, gap in ((1, 0), (3, 5), (70 if width < 9000 else 5, 8)):
        x = rows_of(torch.Generator().manual_seed(width + rows), rows, width, TYPES[dtype], gap)
        say(f"quantize_mx4 {rows} x {width} {dtype} gap {gap}")
        q, s = nm.nm_quantize_mx4(on_gpu(x, width))
        want, scales = round_ref(x[:, :width])
        assert q.shape == (rows, blocks(width) * 16) and s.shape == (rows, blocks(width))
        assert torch.equal(s.cpu().long(), scales) and same(values_of(q, s, width), want)
        assert (values_of(q, s, blocks(width) * 32)[:, width:] == 0).all()
        for t in TYPES.values():
            y = nm.nm_dequantize_mx4(q, s, width, t)
            assert y.dtype == t and same(y.cpu().double(), want)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("width", WIDTHS)
def test_norm(width, dtype):
    g = torch.Generator().manual_seed(width)
    for i, (rows, gap) in enumerate(((1, 0), (3, 5), (70 if width < 9000 else 5, 8))):
        x, r = rows_of(g, rows, width, TYPES[dtype], gap), rows_of(g, rows, width, TYPES[dtype]) if i != 1 else None
        gamma = 1.0 + 0.1 * torch.randn(width, generator=g) if i != 2 else None
        say(f"rmsnorm_mx4 {rows} x {width} {dtype} gap {gap}")
        q, s, h = nm.nm_rmsnorm_mx4(on_gpu(x, width), None if gamma is None else gamma.cuda(), None if r is None else r.cuda(), 1e-6)
        v, want_h = norm_ref(x[:, :width], r, gamma, 1e-6)
        want, scales = round_ref(v)
        assert torch.equal(s.cpu().long(), scales) and same(values_of(q, s, width), want)
        assert (h is None) == (r is None)
        if h is not None:
            assert h.dtype == TYPES[dtype] and torch.equal(h.cpu(), want_h.to(TYPES[dtype]))


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("width", [7, 8, 9, 4097, 4104, 5001, 8185, 8192, 8193, 12000, 16383, 16384])
def test_norm_of_many_rows(width, dtype):
    """Rows that fewer threads take than a few rows' would, the stream in place too."""
    g = torch.Generator().manual_seed(width)
    for rows, gap in ((256, 0), (261, 3)):
        x, r = rows_of(g, rows, width, TYPES[dtype], gap), rows_of(g, rows, width, TYPES[dtype], gap)
        gamma = 1.0 + 0.1 * torch.randn(width, generator=g)
        say(f"rmsnorm_mx4 {rows} x {width} {dtype} gap {gap}")
        v, want_h = norm_ref(x[:, :width], r[:, :width], gamma, 1e-6)
        want, scales = round_ref(v)
        xd, rd = on_gpu(x, width), on_gpu(r, width)
        kept = x.cuda()[:, width:]
        for out in (None, xd):
            q, s, h = nm.nm_rmsnorm_mx4(xd, gamma.cuda(), rd, 1e-6, residual_out=out)
            assert torch.equal(s.cpu().long(), scales) and same(values_of(q, s, width), want)
            assert torch.equal(h.cpu(), want_h.to(TYPES[dtype]))
        if gap:
            assert torch.equal(torch.as_strided(xd, (rows, gap), (width + gap, 1), width), kept)


def test_every_bf16_value():
    """All of them, the ties, the subnormals and those that are not finite, in blocks of nearly equal and of very different magnitudes."""
    bits = torch.arange(65536, dtype=torch.int32)
    for x in (bits.to(torch.int16).view(torch.bfloat16).view(-1, 64), bits.view(32, -1).t().reshape(-1, 32).to(torch.int16).view(torch.bfloat16)):
        say(f"all bf16 values in rows of {x.shape[1]}")
        q, s = nm.nm_quantize_mx4(x.contiguous().cuda())
        want, scales = round_ref(x.double())
        assert torch.equal(s.cpu().long(), scales) and same(values_of(q, s, x.shape[1]), want)
        assert (q.cpu().view(x.shape[0], -1, 16)[scales == 255] == 0).all()
        assert same(nm.nm_dequantize_mx4(q, s, dtype=torch.bfloat16).cpu().double(), want)


def test_borders_in_fp32():
    """Quotients on a border, and the fp32 numbers next to them, under powers of two from the smallest to the largest."""
    b = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9999995, 4.0])
    up, down = torch.nextafter(b, torch.tensor(9.0)), torch.nextafter(b, torch.tensor(0.0))
    unit = torch.cat([b, up.clamp(max=7.9999995), down, torch.tensor([4.0, 0.0, -0.0, 1e-30, 6.0])])
    block = torch.cat([unit, unit.new_zeros(32 - unit.numel())]) if unit.numel() < 32 else unit[:32]
    x = torch.stack([block * 2.0 ** e for e in range(-126, 126)] + [-block * 2.0 ** e for e in (-140, -127, 0, 100)])
    say("borders")
    q, s = nm.nm_quantize_mx4(x.cuda())
    want, scales = round_ref(x.double())
    assert torch.equal(s.cpu().long(), scales) and same(values_of(q, s, 32), want)


def test_values_that_are_not_finite_stay_in_their_block():
    for dtype in TYPES.values():
        x = rows_of(torch.Generator().manual_seed(3), 9, 200, dtype)
        clean, cs = nm.nm_quantize_mx4(x.cuda())
        x[2, 70], x[5, 199], x[7, 0] = math.nan, -math.inf, math.inf
        q, s = nm.nm_quantize_mx4(x.cuda())
        bad = torch.zeros((9, 7), dtype=torch.bool)
        bad[2, 2] = bad[5, 6] = bad[7, 0] = True
        assert torch.equal(s.cpu() == 255, bad) and torch.equal(s.cpu()[~bad], cs.cpu()[~bad])
        q, clean = q.cpu().view(9, 7, 16), clean.cpu().view(9, 7, 16)
        assert (q[bad] == 0).all() and torch.equal(q[~bad], clean[~bad])
        y = nm.nm_dequantize_mx4(q.view(9, -1).cuda(), s, 200)
        assert torch.equal(torch.isnan(y).cpu(), bad.repeat_interleave(32, dim=1)[:, :200])


def test_norms_of_unusual_rows():
    for dtype in TYPES.values():
        x = rows_of(torch.Generator().manual_seed(4), 8, 300, dtype)
        x[1] = 0
        x[2] *= 1e-30
        x[3] *= 1e30
        x[4, 9] = math.inf
        x[5, 299] = math.nan
        for eps in (0.0, 1e-6):
            q, s, h = nm.nm_rmsnorm_mx4(x.cuda(), eps=eps)
            assert h is None
            want, scales = round_ref(norm_ref(x, None, None, eps)[0])
            assert torch.equal(s.cpu().long(), scales) and same(values_of(q, s, 300), want)
            assert torch.isnan(values_of(q, s, 300)[5]).all()


def test_outputs_in_place_and_strided():
    g = torch.Generator().manual_seed(5)
    for dtype in TYPES.values():
        x, r = rows_of(g, 40, 700, dtype).cuda(), rows_of(g, 40, 700, dtype).cuda()
        q0, s0, h0 = nm.nm_rmsnorm_mx4(x, None, r)
        for out in (x.clone(), r.clone()):
            a, b = (out, r) if torch.equal(out, x) else (x, out)
            q, s, h = nm.nm_rmsnorm_mx4(a, None, b, residual_out=out)
            assert h is out and torch.equal(h, h0) and torch.equal(q, q0) and torch.equal(s, s0)
        wide_q = torch.full((40, 22 * 16 + 48), 0x5a, dtype=torch.uint8, device="cuda")
        wide_s = torch.full((40, 29), 0x5a, dtype=torch.uint8, device="cuda")
        q, s = nm.nm_quantize_mx4(x, wide_q[:, 16:16 + 352], wide_s[:, 3:25])
        q1, s1 = nm.nm_quantize_mx4(x)
        assert torch.equal(q, q1) and torch.equal(s, s1)
        assert (wide_q[:, :16] == 0x5a).all() and (wide_q[:, 368:] == 0x5a).all() and (wide_s[:, :3] == 0x5a).all() and (wide_s[:, 25:] == 0x5a).all()
        wide_y = torch.full((40, 711), 7.0, dtype=dtype, device="cuda")
        y = nm.nm_dequantize_mx4(q, s, y=wide_y[:, 5:705])
        assert same(y.cpu().double(), values_of(q1, s1, 700)) and (wide_y[:, :5] == 7).all() and (wide_y[:, 705:] == 7).all()


def test_any_codes_are_read():
    q, s = random_mx4(torch.Generator().manual_seed(6), (50, 333), 0, 256)
    y = nm.nm_dequantize_mx4(q.cuda(), s.cuda(), 333)
    want = values_of(q, s, 333)
    want = torch.where(want.abs() > torch.finfo(torch.float32).max, torch.copysign(torch.tensor(math.inf, dtype=torch.float64), want), want)
    assert same(y.cpu().double(), want)


def test_more_axes_no_rows_and_one_row_repeated():
    x = rows_of(torch.Generator().manual_seed(7), 6, 96, torch.float32).cuda()
    q, s = nm.nm_quantize_mx4(x)
    q3, s3 = nm.nm_quantize_mx4(x.view(2, 3, 96))
    assert q3.shape == (2, 3, 48) and s3.shape == (2, 3, 3) and torch.equal(q3.view(6, 48), q) and torch.equal(s3.view(6, 3), s)
    assert nm.nm_dequantize_mx4(q3, s3).shape == (2, 3, 96)
    q0, s0 = nm.nm_quantize_mx4(x[:0])
    assert q0.shape == (0, 48) and s0.shape == (0, 3) and nm.nm_dequantize_mx4(q0, s0).shape == (0, 96)
    qe, se = nm.nm_quantize_mx4(x[:1].expand(5, 96))
    assert torch.equal(qe, q[:1].expand(5, 48)) and torch.equal(se, s[:1].expand(5, 3))


def test_another_stream_and_a_graph():
    x, r = (rows_of(torch.Generator().manual_seed(i), 64, 1000, torch.bfloat16).cuda() for i in (8, 9))
    want = nm.nm_rmsnorm_mx4(x, None, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = nm.nm_rmsnorm_mx4(x, None, r, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    x0, r0 = x.clone(), r.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = nm.nm_rmsnorm_mx4(x, None, r)
        back = nm.nm_dequantize_mx4(out[0], out[1], 1000)
    for i in range(4):
        x.copy_(x0 * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        want = nm.nm_rmsnorm_mx4(x, None, r)
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and torch.equal(back, nm.nm_dequantize_mx4(want[0], want[1], 1000))
    assert torch.equal(r, r0)
