"""Products in MX4 where their kernels change: long rows, which need their scales in several parts, wide matrices of few rows, many
experts, strides and weights past 32 bits, calls on two streams at once."""
import pytest
import torch

from paper_2507_17301_amd import binding as nm
from gpu_util import say
from mx4_util import blocks, check_close, check_rounded, product_ref, random_mx4, rows_of, values_of
from test_gpu_experts import check_route, grouped_ref, groups_of

pytestmark = pytest.mark.gpu


def check(y, ref):
    if isinstance(y, tuple):
        check_rounded(y[0], y[1], *ref)
    else:
        check_close(y, *ref)


# tall: many workgroups, so that the larger tiles are the faster ones
@pytest.mark.parametrize("rows,k,n", [(10, 65536, 70), (40, 16384, 100), (70, 6145, 70), (130, 13000, 300), (100, 65536, 40), (2500, 6500, 2700)])
@pytest.mark.parametrize("gated", [False, True])
def test_long_rows(rows, k, n, gated):
    g = torch.Generator().manual_seed(rows + k)
    n = n // 2 * 2 if gated else n
    q, s = random_mx4(g, (rows, k))
    w, ws = random_mx4(g, (n, k), 110, 122)
    say(f"linear_mx4 {rows} x {k} x {n} gated {gated}")
    h = nm.nm_mx4_pack(w.cuda(), ws.cuda(), k, gated=gated)
    ref = product_ref(values_of(q, s, k), values_of(w, ws, k), gated=gated)
    y = nm.nm_linear_mx4(q.cuda(), s.cuda(), h, dtype=torch.float32)
    check(y, ref)
    check(nm.nm_linear_mx4(q.cuda(), s.cuda(), h, rounded=True), ref)
    # the last block of a row: a NaN there is that row's alone
    s[rows // 2, -1] = 255
    z = nm.nm_linear_mx4(q.cuda(), s.cuda(), h, dtype=torch.float32)
    rest = torch.arange(rows) != rows // 2
    assert torch.isnan(z[rows // 2]).all() and torch.equal(z[rest], y[rest])


# the smallest sizes whose tiles fill more than the chip once, and some that fill it several times; widths at the ends of blocks, words of scales, steps
@pytest.mark.parametrize("rows,n", [(1025, 1100), (1153, 1030), (4100, 2600)])
@pytest.mark.parametrize("k", [97, 128, 255, 256, 257, 512, 513, 1037])
@pytest.mark.parametrize("gated", [False, True])
def test_tiles(rows, n, k, gated):
    g = torch.Generator().manual_seed(rows + k)
    q, s = random_mx4(g, (rows, k))
    w, ws = random_mx4(g, (n, k), 110, 122)
    bias = torch.randn(n, generator=g) if k % 2 else None
    say(f"linear_mx4 {rows} x {k} x {n} gated {gated}")
    h = nm.nm_mx4_pack(w.cuda(), ws.cuda(), k, gated=gated)
    b = None if bias is None else bias.cuda()
    ref = product_ref(values_of(q, s, k), values_of(w, ws, k), bias, gated=gated)
    y = nm.nm_linear_mx4(q.cuda(), s.cuda(), h, b, dtype=torch.float32)
    check(y, ref)
    check(nm.nm_linear_mx4(q.cuda(), s.cuda(), h, b), ref)
    check(nm.nm_linear_mx4(q.cuda(), s.cuda(), h, b, rounded=True), ref)
    if not gated:
        r = torch.randn((rows, n), generator=g).bfloat16()
        check(nm.nm_linear_mx4(q.cuda(), s.cuda(), h, b, r.cuda()), product_ref(values_of(q, s, k), values_of(w, ws, k), bias, r))
    # a row that is not a number touches no other; nor do codes past the width
    bad = s.clone()
    bad[3, 0] = bad[rows - 1, -1] = 255
    z = nm.nm_linear_mx4(q.cuda(), bad.cuda(), h, b, dtype=torch.float32)
    rest = torch.ones(rows, dtype=torch.bool)
    rest[3] = rest[rows - 1] = False
    assert torch.isnan(z[~rest]).all() and torch.equal(z[rest], y[rest])
    if k % 32:
        q[:, (k + 1) // 2:] = 0x77
        assert torch.equal(nm.nm_linear_mx4(q.cuda(), s.cuda(), h, b, dtype=torch.float32), y)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows", [1, 16, 17, 32, 33, 64, 65])
def test_few_rows_of_wide_matrices(rows, gated):
    g = torch.Generator().manual_seed(rows)
    k, n = 128, 41000        # (more than 640 groups of 64 channels)
    q, s = random_mx4(g, (rows, k))
    w, ws = random_mx4(g, (n, k), 110, 122)
    say(f"linear_mx4 {rows} x {k} x {n} gated {gated}")
    h = nm.nm_mx4_pack(w.cuda(), ws.cuda(), k, gated=gated)
    ref = product_ref(values_of(q, s, k), values_of(w, ws, k), gated=gated)
    for dtype in (torch.float32, torch.bfloat16):
        check(nm.nm_linear_mx4(q.cuda(), s.cuda(), h, dtype=dtype), ref)
    check(nm.nm_linear_mx4(q.cuda(), s.cuda(), h, rounded=True), ref)


@pytest.mark.parametrize("experts,entries,k,n,kind", [(64, 511, 300, 515, "ragged"), (64, 640, 300, 515, "ragged"), (130, 1500, 160, 65, "ragged"),
                                                      (130, 1500, 160, 65, "one"), (1024, 2000, 128, 40, "ragged"), (1024, 9000, 128, 40, "ragged"),
                                                      (1024, 9000, 128, 40, "one"), (3, 200, 7000, 40, "ragged"), (9, 20000, 64, 40, "ragged"), (9, 20000, 160, 40, "ragged")])
@pytest.mark.parametrize("gated", [False, True])
def test_many_experts_of_few_rows(experts, entries, k, n, kind, gated):
    g = torch.Generator().manual_seed(experts + entries + k)
    n = n // 2 * 2 if gated else n
    offsets = groups_of(g, experts, entries, kind)
    w, ws = random_mx4(g, (experts, n, k), 110, 122)
    tokens = entries // 2
    q, s = random_mx4(g, (tokens, k))
    index = torch.randint(0, tokens, (entries,), generator=g, dtype=torch.int32)
    say(f"experts_mx4 {experts} x {entries} x {k} x {n} {kind} gated {gated}")
    h = nm.nm_mx4_pack(w.cuda(), ws.cuda(), k, gated=gated)
    ref = grouped_ref(values_of(q, s, k)[index.long()], offsets, values_of(w, ws, k), None, gated)
    args = q.cuda(), s.cuda(), h, offsets.cuda(), index.cuda()
    check(nm.nm_experts_mx4(*args, dtype=torch.float32), ref)
    check(nm.nm_experts_mx4(*args, rounded=True), ref)
    # the same rows taken beforehand
    direct = nm.nm_experts_mx4(q[index.long()].cuda(), s[index.long()].cuda(), h, offsets.cuda(), dtype=torch.float32)
    check(direct, ref)


@pytest.mark.parametrize("rows", [40, 300])
def test_rows_further_apart_than_32_bits(rows):
    """Rows at the largest stride: tensors of 5 GiB."""
    g = torch.Generator().manual_seed(rows)
    k, n, ld = 320, 70, 1 << 24
    q, s = random_mx4(g, (rows, k))
    h = nm.nm_mx4_pack(*(v.cuda() for v in random_mx4(g, (n, k), 110, 122)))
    say(f"linear_mx4 {rows} x {k} x {n}, stride {ld}")
    want = nm.nm_linear_mx4(q.cuda(), s.cuda(), h)
    b = blocks(k)
    wide = torch.empty(rows * ld, dtype=torch.uint8, device="cuda").view(rows, ld)
    wide[:, :b * 16], wide[:, 4096:4096 + b] = q.cuda(), s.cuda()
    out = wide.view(torch.bfloat16)[:, 8192:8192 + n]
    nm.nm_linear_mx4(wide[:, :b * 16], wide[:, 4096:4096 + b], h, y=out)
    assert torch.equal(out, want)
    x = wide.view(torch.float32)[:, 65536:65536 + k]
    x.copy_(rows_of(g, rows, k, torch.float32))
    flat = x.contiguous()
    for a, c in zip(nm.nm_rmsnorm_mx4(x, None, x, residual_out=x), nm.nm_rmsnorm_mx4(flat, None, flat)):
        assert torch.equal(a, c)
    nm.nm_quantize_mx4(x, q=wide[:, :b * 16], scales=wide[:, 4096:4096 + b])
    assert torch.equal(nm.nm_dequantize_mx4(wide[:, :b * 16], wide[:, 4096:4096 + b], k), nm.nm_dequantize_mx4(*nm.nm_quantize_mx4(x.contiguous()), k))


def test_weights_of_more_than_32_bits():
    """4.6 GB of packed weights, of which the last expert's rows want the last."""
    g = torch.Generator().manual_seed(3)
    experts, n, k = 1024, 4096, 2112
    w = torch.randint(0, 256, (experts, n, k // 2), dtype=torch.uint8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    ws = torch.randint(110, 122, (experts, n, k // 32), dtype=torch.uint8, device="cuda")
    h = nm.nm_mx4_pack(w, ws)
    last, scales = w[-1, -64:].cpu(), ws[-1, -64:].cpu()
    del w, ws
    for rows in (5, 90):
        q, s = random_mx4(g, (rows, k))
        offsets = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
        offsets[-1] = rows
        say(f"experts_mx4 {experts} x {rows} x {k} x {n}")
        y = nm.nm_experts_mx4(q.cuda(), s.cuda(), h, offsets, dtype=torch.float32)
        check(y[:, -64:], product_ref(values_of(q, s, k), values_of(last, scales, k)))
    h.free()


def test_two_streams_at_once():
    g = torch.Generator().manual_seed(8)
    experts, tokens, width, k = 12, 300, 640, 3
    x, logits = rows_of(g, tokens, width, torch.bfloat16).cuda(), torch.randn((tokens, experts), generator=g).cuda()
    h = nm.nm_mx4_pack((torch.randn((experts, 512, width), generator=g) / 25).cuda())

    def run():
        to = nm.nm_route(logits, k)
        q, s = nm.nm_quantize_mx4(x)
        return nm.nm_combine(nm.nm_experts_mx4(q, s, h, to.offsets, to.rows), to.slots, to.weights)

    want = run()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(run())
    torch.cuda.synchronize()
    for y in got:
        assert torch.equal(y, want)
    with_stream = nm.nm_rmsnorm_mx4(x, stream=streams[0])
    streams[0].synchronize()
    assert all(torch.equal(a, b) for a, b in zip(with_stream[:2], nm.nm_rmsnorm_mx4(x)[:2]))


def test_graphs_with_their_own_workspaces():
    """Two captured graphs of the same calls, replayed in turn and with eager calls between them."""
    g = torch.Generator().manual_seed(9)
    experts, tokens = 40, 700
    logits = [torch.randn((tokens, experts), generator=g).cuda() for _ in range(2)]
    graphs, outs = [], []
    nm.nm_route(logits[0], 4)
    for l in logits:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(nm.nm_route(l, 4))
        graphs.append(graph)
    for i in range(4):
        for l in logits:
            l.copy_(l.roll(1, dims=1))
        for graph in graphs[:: 1 if i % 2 else -1]:
            graph.replay()
        eager = [nm.nm_route(l, 4) for l in logits]
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert all(torch.equal(s, t) for s, t in zip(a, b))


@pytest.mark.parametrize("tokens", [64, 65, 200])
def test_routing_with_as_many_choices_as_there_may_be(tokens):
    g = torch.Generator().manual_seed(tokens)
    check_route(torch.randn((tokens, 100), generator=g), 64)
    check_route(torch.randn((tokens, 64), generator=g).bfloat16(), 64, normalise=False)
    check_route(torch.randn((tokens, 1024), generator=g).bfloat16(), 64, ld=3)
