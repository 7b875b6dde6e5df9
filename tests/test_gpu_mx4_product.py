"""Products in MX4 and the feed-forward layer against their formulas in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2507_17301_amd import binding as nm
from paper_2507_17301_amd.feedforward import FeedForwardMX4
from gpu_util import say
from mx4_util import blocks, check_close, check_rounded, product_ref, random_mx4, round_ref, rows_of, values_of

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# rows: one, the ends of 16-row blocks and of the few-row kernels, past the tile kernels' first tile
ROWS = [1, 2, 15, 16, 17, 32, 33, 64, 65, 100, 128, 129, 256, 257, 300, 515]
# widths and channels: one, odd ones, the ends of blocks, steps, groups and tiles
SIZES = [(1, 1), (32, 3), (63, 64), (64, 65), (255, 16), (256, 130), (257, 31), (512, 256), (1037, 75), (1024, 514), (2064, 100)]


def inputs(rows, k, n, seed):
    g = torch.Generator().manual_seed(seed)
    q, s = random_mx4(g, (rows, k))
    w, ws = random_mx4(g, (n, k), 110, 122)
    return q, s, w, ws, torch.randn(n, generator=g)


def check(y, ref):
    if isinstance(y, tuple):
        check_rounded(y[0], y[1], *ref)
    else:
        check_close(y, *ref)


@pytest.mark.parametrize("out", ["bf16", "f32", "mx4"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("k,n", SIZES)
def test_product(k, n, gated, out):
    n = 2 * n if gated else n
    for i, rows in enumerate(ROWS):
        q, s, w, ws, bias = inputs(rows, k, n, 100 * k + rows)
        bias = bias if i % 2 else None
        say(f"linear_mx4 {rows} x {k} x {n} gated {gated} {out} bias {bias is not None}")
        h = nm.nm_mx4_pack(w.cuda(), ws.cuda(), k, gated=gated)
        t = TYPES.get(out)
        r = torch.randn((rows, n), generator=torch.Generator().manual_seed(rows)).to(t) if i % 3 == 0 and not gated and t else None
        y = nm.nm_linear_mx4(q.cuda(), s.cuda(), h, None if bias is None else bias.cuda(), None if r is None else r.cuda(), t, rounded=t is None)
        torch.cuda.synchronize()
        if t:
            assert y.shape == (rows, h.outs) and y.dtype == t
        check(y, product_ref(values_of(q, s, k), values_of(w, ws, k), bias, r, gated))


@pytest.mark.parametrize("rows,k,n", [(3, 300, 70), (40, 1024, 200), (90, 1000, 130), (700, 512, 1100), (2500, 256, 2700), (1111, 1100, 5000), (300, 9000, 300)])
@pytest.mark.parametrize("gated", [False, True])
def test_larger_products_with_their_rows_in_place(rows, k, n, gated):
    n = 2 * n if gated else n
    q, s, w, ws, bias = inputs(rows, k, n, rows)
    say(f"linear_mx4 {rows} x {k} x {n} gated {gated}, strided")
    h = nm.nm_mx4_pack(w.cuda(), ws.cuda(), k, gated=gated)
    ref = product_ref(values_of(q, s, k), values_of(w, ws, k), bias, None, gated)
    y0 = nm.nm_linear_mx4(q.cuda(), s.cuda(), h, bias.cuda())
    check(y0, ref)
    check(nm.nm_linear_mx4(q.cuda(), s.cuda(), h, bias.cuda(), rounded=True), ref)
    b = blocks(k)
    qw = torch.full((rows, 16 * b + 48), 0x77, dtype=torch.uint8, device="cuda")       # rows of wider tensors into rows of another
    sw = torch.full((rows, b + 3), 0xff, dtype=torch.uint8, device="cuda")
    qw[:, 16:16 + 16 * b], sw[:, 1:1 + b] = q.cuda(), s.cuda()
    yw = torch.full((rows, h.outs + 7), 4.0, dtype=torch.bfloat16, device="cuda")
    y = nm.nm_linear_mx4(qw[:, 16:16 + 16 * b], sw[:, 1:1 + b], h, bias.cuda(), y=yw[:, 3:3 + h.outs])
    assert torch.equal(y, y0) and (yw[:, :3] == 4).all() and (yw[:, 3 + h.outs:] == 4).all()
    if not gated:                            # the residual stream updated in place
        stream = torch.randn((rows, n), device="cuda")
        ref = product_ref(values_of(q, s, k), values_of(w, ws, k), None, stream.cpu())
        y = nm.nm_linear_mx4(q.cuda(), s.cuda(), h, None, stream, y=stream)
        assert y is stream
        check(y, ref)


def test_what_lies_past_the_width_changes_nothing():
    """Codes past the width in the last block of rows and weights, and the bytes behind a row's."""
    for rows in (5, 40, 200):
        q, s, w, ws, _ = inputs(rows, 300, 70, rows)
        qz, wz = q.clone(), w.clone()
        for t in (qz, wz):
            t[:, 300 // 2:] = 0
        a = nm.nm_linear_mx4(q.cuda(), s.cuda(), nm.nm_mx4_pack(w.cuda(), ws.cuda(), 300), dtype=torch.float32)
        b = nm.nm_linear_mx4(qz.cuda(), s.cuda(), nm.nm_mx4_pack(wz.cuda(), ws.cuda(), 300), dtype=torch.float32)
        assert torch.equal(a, b)


@pytest.mark.parametrize("gated", [False, True])
def test_a_row_that_is_not_a_number_touches_no_other(gated):
    for rows in (4, 30, 70, 300):
        q, s, w, ws, bias = inputs(rows, 1056, 450, 9)
        h = nm.nm_mx4_pack(w.cuda(), ws.cuda(), gated=gated)
        whole = nm.nm_linear_mx4(q.cuda(), s.cuda(), h, bias.cuda(), dtype=torch.float32)
        again = nm.nm_linear_mx4(q.cuda(), s.cuda(), h, bias.cuda(), dtype=torch.float32)
        assert torch.equal(whole, again)
        for at in ((3, 0), (rows - 1, 32)):
            bad = s.clone()
            bad[at] = 255
            y = nm.nm_linear_mx4(q.cuda(), bad.cuda(), h, bias.cuda(), dtype=torch.float32)
            rest = torch.arange(rows) != at[0]
            assert torch.isnan(y[at[0]]).all() and torch.equal(y[rest], whole[rest])
            _, ys = nm.nm_linear_mx4(q.cuda(), bad.cuda(), h, bias.cuda(), rounded=True)
            assert (ys[at[0]] == 255).all() and (ys[rest] != 255).all()


def test_powers_far_from_one():
    """The smallest and the largest scales: what leaves fp32's range does so as the formula in fp32 would."""
    q, s, w, ws, _ = inputs(20, 128, 40, 12)
    for a, b in ((1, 250), (250, 1), (0, 200), (60, 60)):
        s[:], ws[:] = a, b
        y = nm.nm_linear_mx4(q.cuda(), s.cuda(), nm.nm_mx4_pack(w.cuda(), ws.cuda()), dtype=torch.float32)
        ref, bound = product_ref(values_of(q, s, 128), values_of(w, ws, 128))
        check_close(y, ref, bound + 128 * 2.0 ** -126)   # (products below fp32's normal numbers may count as zeros)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_packing(dtype):
    for n in (2, 62, 64, 130):
        for k in (1, 17, 128, 333):
            for gated in (False, True):
                g = torch.Generator().manual_seed(n + k)
                w = rows_of(g, n, k, TYPES[dtype], gap=3)[:, :k]
                h = nm.nm_mx4_pack(w.cuda(), gated=gated)
                assert (h.experts, h.channels, h.width) == (1, n, k)
                a, t = (torch.from_numpy(v)[0] for v in nm.nm_mx4_export(h))
                want, scales = round_ref(w.double())
                assert torch.equal(t.long(), scales) and torch.equal(values_of(a, t, k) + 0.0, want + 0.0)
                h4 = nm.nm_mx4_pack(a.cuda(), t.cuda(), k, gated=gated)
                a4, t4 = nm.nm_mx4_export(h4)
                assert np.array_equal(a4[0], a.numpy()) and np.array_equal(t4[0], t.numpy())
                h4.free()
                h4.free()
    w = torch.randn((6, 40)).to(TYPES[dtype])
    for v in (math.nan, math.inf):
        w[4, 39] = v
        with pytest.raises(nm.NMError) as e:
            nm.nm_mx4_pack(w.cuda())
        assert e.value.code == nm.NM_ERR_ARG and "finite" in str(e.value)


def test_no_rows_more_axes_and_one_row_repeated():
    q, s, w, ws, bias = inputs(6, 96, 40, 3)
    q, s = q.cuda(), s.cuda()
    h = nm.nm_mx4_pack(w.cuda(), ws.cuda())
    assert nm.nm_linear_mx4(q[:0], s[:0], h).shape == (0, 40)
    y = nm.nm_linear_mx4(q, s, h)
    y3 = nm.nm_linear_mx4(q.view(2, 3, 48), s.view(2, 3, 3), h)
    assert y3.shape == (2, 3, 40) and torch.equal(y3.view(6, 40), y)
    for rows in (9, 100):
        ye = nm.nm_linear_mx4(q[2:3].expand(rows, 48), s[2:3].expand(rows, 3), h)
        assert torch.equal(ye, ye[:1].expand(rows, 40))
        check(ye[:1], product_ref(values_of(q[2:3], s[2:3], 96), values_of(w, ws, 96)))


def test_refusals():
    q, s, w, ws, bias = (t.cuda() for t in inputs(4, 96, 40, 3))
    h, hg, he = nm.nm_mx4_pack(w, ws), nm.nm_mx4_pack(w, ws, gated=True), nm.nm_mx4_pack(w.view(2, 20, 48), ws.view(2, 20, 3))
    r = torch.zeros((4, 40), dtype=torch.bfloat16, device="cuda")
    shifted = torch.zeros((4 * 48 + 8,), dtype=torch.uint8, device="cuda")[8:].view(4, 48)
    for call, code in ((lambda: nm.nm_linear_mx4(q, s, hg, residual=r[:, :20].contiguous()), nm.NM_ERR_UNSUPPORTED),
                       (lambda: nm.nm_linear_mx4(q, s, he), nm.NM_ERR_UNSUPPORTED),
                       (lambda: nm.nm_linear_mx4(shifted, s, h), nm.NM_ERR_ARG),
                       (lambda: nm.nm_mx4_pack(w, ws.clone().fill_(255)), nm.NM_ERR_ARG)):
        with pytest.raises(nm.NMError) as e:
            call()
        assert e.value.code == code
    for call in (lambda: nm.nm_linear_mx4(q[:, :32], s[:, :2], h), lambda: nm.nm_linear_mx4(q, s[:, :2], h), lambda: nm.nm_linear_mx4(q[:, :40], s, h),
                 lambda: nm.nm_linear_mx4(q, s, h, bias=bias[:39]), lambda: nm.nm_linear_mx4(q, s, h, y=r[:, :39]),
                 lambda: nm.nm_linear_mx4(q, s, h, y=r, y_scales=s), lambda: nm.nm_mx4_pack(w, ws, width=64)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        nm.nm_linear_mx4(q.to(torch.int8), s, h)
    h.free()
    with pytest.raises(nm.NMError):
        nm.nm_linear_mx4(q, s, h)


def test_layer_and_graph():
    g = torch.Generator().manual_seed(21)
    width, hidden = 320, 416
    gate, up, down = (torch.randn(s, generator=g) / s[1] ** 0.5 for s in ((hidden, width), (hidden, width), (width, hidden)))
    gamma = 1.0 + 0.1 * torch.randn(width, generator=g)
    layer = FeedForwardMX4.from_float(gamma.cuda(), gate.cuda(), up.cuda(), down.cuda())
    w1, w2 = round_ref(torch.cat([gate, up]))[0], round_ref(down)[0]
    for dtype in TYPES.values():
        for rows in (1, 20, 200):
            x, r = rows_of(g, rows, width, dtype), rows_of(g, rows, width, dtype)
            say(f"FeedForwardMX4 {rows} rows {dtype}")
            h = x.float() + r.float()
            n = (1.0 / torch.sqrt((h.double() ** 2).mean(dim=1, keepdim=True) + 1e-6)).float()
            v = round_ref(h * n * gamma)[0]
            # what the second product gets is the kernel's own rounding, held to its bound
            q, s, stream = nm.nm_rmsnorm_mx4(x.cuda(), gamma.cuda(), r.cuda())
            q, s = nm.nm_linear_mx4(q, s, layer.up, rounded=True)
            check_rounded(q, s, *product_ref(v, w1, gated=True))
            y = layer(x.cuda(), r.cuda())
            assert y.dtype == dtype
            check_close(y, *product_ref(values_of(q, s, hidden), w2, None, stream.cpu()))
            xd, rd = x.cuda(), r.cuda()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = layer(xd, rd)
            for i in range(3):
                xd.copy_((x.float() * (1 + i)).to(dtype))
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(out, layer(xd, rd))


def test_a_handle_freed_under_capture():
    g = torch.Generator().manual_seed(77)
    q, s = nm.nm_quantize_mx4(rows_of(g, 3, 256, torch.float32).cuda())
    h, other = (nm.nm_mx4_pack(rows_of(g, 128, 256, torch.float32).cuda()) for _ in range(2))
    ref = nm.nm_linear_mx4(q, s, h, dtype=torch.float32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other.free()
        y = nm.nm_linear_mx4(q, s, h, dtype=torch.float32)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ref)
