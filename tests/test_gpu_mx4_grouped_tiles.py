"""The tile kernels of products in MX4 grouped by expert, and the same kernels of one matrix where long rows, rows and weights past 32 bits,
other streams and graphs come in.  The sizes are those of mx4_cases.py, whose kernels tests/test_mx4_launches.py asserts."""
import pytest
import torch

import mx4_cases as cases
from paper_2507_17301_amd import binding as nm
from paper_2507_17301_amd.feedforward import ExpertsMX4, FeedForwardMX4
from gpu_util import say
from mx4_util import U, blocks, check_close, check_rounded, product_ref, random_mx4, round_ref, rows_of, values_of
from test_gpu_experts import TYPES, grouped_ref, groups_of, route_ref

pytestmark = pytest.mark.gpu


def check(y, ref):
    if isinstance(y, tuple):
        check_rounded(y[0], y[1], *ref)
    else:
        check_close(y, *ref)


def _grouped(g, experts, entries, k, n, gated, kind="ragged"):
    """(offsets, handle, weights' values, biases)"""
    offsets = groups_of(g, experts, entries, kind)
    w, ws = random_mx4(g, (experts, n, k), 110, 122)
    return offsets, nm.nm_mx4_pack(w.cuda(), ws.cuda(), k, gated=gated), values_of(w, ws, k), torch.randn((experts, n), generator=g)


def _outputs(q, s, h, offsets, index, bias):
    """fp32, bf16 and MX4."""
    args = q.cuda(), s.cuda(), h, offsets.cuda(), None if index is None else index.cuda(), None if bias is None else bias.cuda()
    return [nm.nm_experts_mx4(*args, dtype=torch.float32), nm.nm_experts_mx4(*args), nm.nm_experts_mx4(*args, rounded=True)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape,size", [(shape, size) for shape in sorted(cases.GROUPED) for size in cases.GROUPED[shape] + [cases.GROUPED_LONG[shape]]])
def test_groups(shape, size, gated):
    experts, entries, k, n = size
    g = torch.Generator().manual_seed(entries + k)
    offsets, h, wv, bias = _grouped(g, experts, entries, k, n, gated)
    for tokens in (None, entries // 4 + 3):
        q, s = random_mx4(g, (tokens or entries, k))
        index = torch.randint(0, tokens, (entries,), generator=g, dtype=torch.int32) if tokens else None
        b = bias if tokens else None
        say(f"experts_mx4 {shape}: {experts} x {entries} x {k} x {n} gated {gated} gather {tokens}")
        x = values_of(q, s, k)
        ref = grouped_ref(x if index is None else x[index.long()], offsets, wv, b, gated)
        for y in _outputs(q, s, h, offsets, index, b):
            check(y, ref)


@pytest.mark.parametrize("kind", ["one", "even"])
@pytest.mark.parametrize("shape", sorted(cases.GROUPED))
def test_one_group_and_even_ones(shape, kind):
    for experts, entries, k, n in cases.GROUPED[shape][:2]:
        g = torch.Generator().manual_seed(entries)
        offsets, h, wv, bias = _grouped(g, experts, entries, k, n, False, kind)
        q, s = random_mx4(g, (entries, k))
        say(f"experts_mx4 {shape}: {experts} x {entries} x {k} x {n} {kind}")
        ref = grouped_ref(values_of(q, s, k), offsets, wv, bias, False)
        for y in _outputs(q, s, h, offsets, None, bias):
            check(y, ref)


@pytest.mark.parametrize("shape", sorted(cases.LONG))
@pytest.mark.parametrize("gated", [False, True])
def test_long_rows_of_one_matrix(shape, gated):
    rows, k, n = cases.LONG[shape]
    g = torch.Generator().manual_seed(rows)
    q, s = random_mx4(g, (rows, k))
    w, ws = random_mx4(g, (n, k), 110, 122)
    say(f"linear_mx4 {shape}: {rows} x {k} x {n} gated {gated}")
    h = nm.nm_mx4_pack(w.cuda(), ws.cuda(), k, gated=gated)
    ref = product_ref(values_of(q, s, k), values_of(w, ws, k), gated=gated)
    y = nm.nm_linear_mx4(q.cuda(), s.cuda(), h, dtype=torch.float32)
    check(y, ref)
    # NaN in the first block, in the last one whose scales are dealt first, in the first dealt later, in the last
    bad = s.clone()
    at = [(1, 0), (rows // 3, 191), (rows // 2, 192), (rows - 1, blocks(k) - 1)]
    for a in at:
        bad[a] = 255
    z = nm.nm_linear_mx4(q.cuda(), bad.cuda(), h, dtype=torch.float32)
    lost = torch.zeros(rows, dtype=torch.bool)
    lost[[a[0] for a in at]] = True
    assert torch.isnan(z[lost]).all() and torch.equal(z[~lost], y[~lost])


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape", sorted(cases.GROUPED))
def test_indices_out_of_range(shape, gated):
    """A row that there is not gives a row of NaN and touches no other; long rows too, whose scales are dealt out twice."""
    for experts, entries, k, n in (cases.GROUPED[shape][0], cases.GROUPED_LONG[shape]):
        g = torch.Generator().manual_seed(entries + 1)
        offsets, h, _, bias = _grouped(g, experts, entries, k, n, gated, "even")
        tokens = entries // 3
        q, s = random_mx4(g, (tokens, k))
        index = torch.randint(0, tokens, (entries,), generator=g, dtype=torch.int32)
        say(f"experts_mx4 {shape}: {experts} x {entries} x {k} x {n} gated {gated}, indices out of range")
        good = _outputs(q, s, h, offsets, index, bias)
        lost = torch.zeros(entries, dtype=torch.bool)
        for at, value in ((0, -1), (5, tokens), (int(offsets[1]) - 1, 2 ** 31 - 1), (int(offsets[1]), -2 ** 31), (entries - 1, tokens + 7)):
            index[at], lost[at] = value, True
        bad = _outputs(q, s, h, offsets, index, bias)
        for a, b in zip(good[:2], bad[:2]):
            assert torch.isnan(b[lost]).all() and torch.equal(a[~lost], b[~lost])
        assert (bad[2][1][lost] == 255).all() and (bad[2][0][lost] == 0).all()
        assert torch.equal(bad[2][0][~lost], good[2][0][~lost]) and torch.equal(bad[2][1][~lost], good[2][1][~lost])


@pytest.mark.parametrize("shape", sorted(cases.GROUPED))
def test_offsets_out_of_range(shape):
    """Offsets past the ends count as the ends, a group that ends before it begins as empty."""
    experts, entries, k, n = 4, {"128 rows": 8000, "64 rows": 1200}[shape], 300, 1030
    g = torch.Generator().manual_seed(entries)
    w, ws = random_mx4(g, (experts, n, k), 110, 122)
    h = nm.nm_mx4_pack(w.cuda(), ws.cuda(), k)
    q, s = (v.cuda() for v in random_mx4(g, (entries, k)))
    half = entries // 2
    say(f"experts_mx4 {shape}: offsets out of range")

    def run(offsets):
        y = torch.full((entries, n), 5.0, device="cuda")
        return nm.nm_experts_mx4(q, s, h, torch.tensor(offsets, dtype=torch.int32, device="cuda"), y=y)
    good = run([0, half, half, half, entries])
    assert (good != 5).any(dim=1).all()
    keep = torch.ones(entries, dtype=torch.bool)
    keep[half - 3:half] = False                          # (those three rows are the third group's, too)
    assert torch.equal(run([-7, half, half - 3, half, entries + 1000])[keep], good[keep])
    assert torch.equal(run([-2 ** 31, half, half, half, 2 ** 31 - 1]), good)
    assert (run([0] * 5) == 5).all() and (run([entries] * 5) == 5).all() and (run([2 ** 31 - 1] * 5) == 5).all() and (run([entries, 0, 0, 0, 0]) == 5).all()


@pytest.mark.parametrize("entries", [1000, 8000])
def test_offsets_that_fall(entries):
    """Groups overlap, and may have more tiles than groups side by side could: a value is one group's or is left, and nothing else is written."""
    experts, k, n = 5, 300, 1030
    g = torch.Generator().manual_seed(entries)
    h = nm.nm_mx4_pack(*(v.cuda() for v in random_mx4(g, (experts, n, k), 110, 122)), k)
    q, s = (v.cuda() for v in random_mx4(g, (entries, k)))
    say(f"experts_mx4 {entries} entries, offsets that fall")

    def run(offsets):
        y = torch.full((entries + 2, n + 2), 5.0, device="cuda")
        nm.nm_experts_mx4(q, s, h, torch.tensor(offsets, dtype=torch.int32, device="cuda"), y=y[1:1 + entries, 1:1 + n])
        return y
    alone = [run([0] * (e + 1) + [entries] * (experts - e)) for e in range(experts)]   # all rows by expert e
    for offsets in ([0, entries * 9 // 10, entries // 10, entries, 0, entries], [entries, 0, entries - 2, 0, entries - 1, 3]):
        y = run(offsets)
        fits = y == 5
        for e in range(experts):
            begin, end = 1 + offsets[e], 1 + max(offsets[e], offsets[e + 1])
            fits[begin:end] |= y[begin:end] == alone[e][begin:end]
        assert bool(fits.all())


@pytest.mark.parametrize("shape", sorted(cases.GROUPED))
def test_rows_in_no_group_are_left_as_they_were(shape):
    experts, entries, k, n = cases.GROUPED[shape][0]
    g = torch.Generator().manual_seed(entries + 2)
    w, ws = random_mx4(g, (experts, n, k), 110, 122)
    h = nm.nm_mx4_pack(w.cuda(), ws.cuda(), k)
    q, s = (v.cuda() for v in random_mx4(g, (entries, k)))
    begin = 3
    offsets = groups_of(g, experts, entries * 2 // 3, "ragged") + begin
    offsets, end = offsets.cuda(), int(offsets[-1])
    say(f"experts_mx4 {shape}: rows in no group")
    full = nm.nm_experts_mx4(q, s, h, offsets, dtype=torch.float32)
    for t in (torch.float32, torch.bfloat16):
        y = torch.full((entries, n + 6), 5.0, device="cuda", dtype=t)
        nm.nm_experts_mx4(q, s, h, offsets, y=y[:, 3:3 + n])
        assert torch.equal(y[begin:end, 3:3 + n], full[begin:end].to(t)) and (y[:begin] == 5).all() and (y[end:] == 5).all()
        assert (y[:, :3] == 5).all() and (y[:, 3 + n:] == 5).all()
    b = blocks(n)
    yq, ys = torch.full((entries, 16 * b + 16), 0x33, dtype=torch.uint8, device="cuda"), torch.full((entries, b + 1), 0x33, dtype=torch.uint8, device="cuda")
    nm.nm_experts_mx4(q, s, h, offsets, y=yq[:, :16 * b], y_scales=ys[:, :b], rounded=True)
    assert all((t[:begin] == 0x33).all() and (t[end:] == 0x33).all() for t in (yq, ys)) and (yq[:, 16 * b:] == 0x33).all() and (ys[:, b] == 0x33).all()
    a, c = nm.nm_experts_mx4(q, s, h, offsets, rounded=True)
    assert torch.equal(yq[begin:end, :16 * b], a[begin:end]) and torch.equal(ys[begin:end, :b], c[begin:end])


# ------------------------------------------------------------------ addresses past 32 bits
def test_rows_further_apart_than_32_bits():
    """Rows at the largest stride, 5 GiB: of one matrix, of two experts, and as many as there may be by index (just under 4 GiB)."""
    ld = 1 << 24
    for kind in ("rows", "entries", "index"):
        *front, k, n = cases.FAR[kind]
        sources, b = front[-1], blocks(k)
        g = torch.Generator().manual_seed(len(kind))
        q, s = (v.cuda() for v in random_mx4(g, (sources, k)))
        wide = torch.empty(sources * ld, dtype=torch.uint8, device="cuda").view(sources, ld)
        wq, wsc = wide[:, :b * 16], wide[:, 4096:4096 + b]
        wq.copy_(q)
        wsc.copy_(s)
        say(f"MX4 tiles, rows {ld} bytes apart: {kind}")
        if kind == "rows":
            h = nm.nm_mx4_pack(*(v.cuda() for v in random_mx4(g, (n, k), 110, 122)), k)
            def run(x, sc, y=None):
                return nm.nm_linear_mx4(x, sc, h, y=y)
        else:
            experts, entries = front[0], front[1]
            h = nm.nm_mx4_pack(*(v.cuda() for v in random_mx4(g, (experts, n, k), 110, 122)), k)
            offsets = groups_of(g, experts, entries, "even").cuda()
            index = torch.randint(0, sources, (entries,), generator=g, dtype=torch.int32).cuda() if kind == "index" else None
            def run(x, sc, y=None):
                return nm.nm_experts_mx4(x, sc, h, offsets, index, y=y)
        want = run(q, s)
        if kind == "index":
            assert torch.equal(run(wq, wsc), want)
        else:
            out = wide.view(torch.bfloat16)[:, 8192:8192 + n]
            run(wq, wsc, out)
            assert torch.equal(out, want)
        del wide, wq, wsc


def test_weights_of_more_than_32_bits():
    """All rows are the last expert's, whose weights lie behind 4 GB of others'."""
    experts, entries, k, n = cases.HEAVY
    g = torch.Generator().manual_seed(3)
    w = torch.randint(0, 256, (experts, n, k // 2), dtype=torch.uint8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    ws = torch.randint(110, 122, (experts, n, k // 32), dtype=torch.uint8, device="cuda")
    h = nm.nm_mx4_pack(w, ws)
    last, scales = w[-1, -64:].cpu(), ws[-1, -64:].cpu()
    del w, ws
    q, s = random_mx4(g, (entries, k))
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    offsets[-1] = entries
    say(f"experts_mx4 {experts} x {entries} x {k} x {n}")
    y = nm.nm_experts_mx4(q.cuda(), s.cuda(), h, offsets, dtype=torch.float32)
    check(y[:, -64:], product_ref(values_of(q, s, k), values_of(last, scales, k)))
    h.free()


# ------------------------------------------------------------------ streams, graphs, layers
@pytest.mark.parametrize("shape", sorted(cases.GROUPED))
def test_graphs_whose_groups_change(shape):
    """Two captured graphs of one handle, replayed in turn on other sizes of groups than those at capture, with eager calls between them."""
    experts, entries, k, n = cases.GROUPED[shape][0]
    g = torch.Generator().manual_seed(entries + 5)
    w, ws = random_mx4(g, (experts, n, k), 110, 122)
    h = nm.nm_mx4_pack(w.cuda(), ws.cuda(), k)
    q, s = (v.cuda() for v in random_mx4(g, (entries // 2, k)))
    say(f"experts_mx4 {shape}: graphs")
    sets = [[groups_of(g, experts, entries, kind).cuda() for kind in kinds] for kinds in (("ragged", "one", "even", "ragged"), ("even", "ragged", "one", "ragged"))]
    indices = [torch.randint(0, entries // 2, (entries,), generator=g, dtype=torch.int32).cuda() for _ in range(4)]
    at = [(v[0].clone(), indices[0].clone()) for v in sets]
    graphs, outs = [], []
    nm.nm_experts_mx4(q, s, h, *at[0])
    for offsets, index in at:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append((nm.nm_experts_mx4(q, s, h, offsets, index), *nm.nm_experts_mx4(q, s, h, offsets, index, rounded=True)))
        graphs.append(graph)
    for i in range(4):
        for (offsets, index), v in zip(at, sets):
            offsets.copy_(v[i])
            index.copy_(indices[i])
        for graph in graphs[:: 1 if i % 2 else -1]:
            graph.replay()
        eager = [(nm.nm_experts_mx4(q, s, h, *a), *nm.nm_experts_mx4(q, s, h, *a, rounded=True)) for a in at]
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert all(torch.equal(x, y) for x, y in zip(a, b)), i


def test_two_streams_at_once():
    experts, entries, k, n = cases.GROUPED["128 rows"][0]
    g = torch.Generator().manual_seed(8)
    offsets, h, _, _ = _grouped(g, experts, entries, k, n, False)
    q, s = (v.cuda() for v in random_mx4(g, (entries, k)))
    offsets = offsets.cuda()
    want = nm.nm_experts_mx4(q, s, h, offsets)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for stream in streams:
        stream.wait_stream(torch.cuda.current_stream())
    say("experts_mx4 on two streams")
    got = [nm.nm_experts_mx4(q, s, h, offsets, stream=stream) for _ in range(8) for stream in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in got)


@pytest.mark.parametrize("experts,k,tokens,width,hidden", cases.EXPERTS_LAYERS)
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_layer_of_experts(experts, k, tokens, width, hidden, dtype):
    dtype = TYPES[dtype]
    g = torch.Generator().manual_seed(tokens)
    (w1, s1), (w2, s2) = random_mx4(g, (experts, 2 * hidden, width), 116, 122), random_mx4(g, (experts, width, hidden), 116, 122)
    layer = ExpertsMX4(nm.nm_mx4_pack(w1.cuda(), s1.cuda(), width, gated=True), nm.nm_mx4_pack(w2.cuda(), s2.cuda(), hidden), k)
    x, r, logits = rows_of(g, tokens, width, dtype), rows_of(g, tokens, width, dtype), torch.randn((tokens, experts), generator=g)
    logits[::9] = -torch.inf                             # padding: the residual stream comes back
    say(f"ExpertsMX4 {experts} experts, {tokens} tokens, {width} x {hidden}, {dtype}")
    _, weights, offsets, rows, slots = route_ref(logits, k)
    end = offsets[-1]
    to = nm.nm_route(logits.cuda(), k)
    q, s = nm.nm_experts_mx4(*nm.nm_quantize_mx4(x.cuda()), layer.up, to.offsets, to.rows, rounded=True)
    check_rounded(q[:end], s[:end], *grouped_ref(round_ref(x.double())[0][rows[:end]], offsets, values_of(w1, s1, width), None, True))
    # what the second product gets is the kernel's own rounding
    y, bound = grouped_ref(values_of(q[:end], s[:end], hidden), offsets, values_of(w2, s2, hidden), None, False)
    pick, open_ = torch.where(slots >= 0, slots, 0), (slots >= 0)[..., None]
    terms = torch.where(open_, weights[..., None] * y[pick], 0.0)
    # the weights: (2 * spread + 8 + experts) u as for the routing; each of the k products and sums, the residual's sum: a rounding
    spread = 2 * float(logits[torch.isfinite(logits)].abs().max())
    size = terms.abs().sum(dim=1) + r.double().abs()
    err = torch.where(open_, weights[..., None] * bound[pick], 0.0).sum(dim=1) + (2 * spread + 8 + experts + k + 2) * U * size
    xd, rd, ld = x.cuda(), r.cuda(), logits.cuda()
    out = layer(xd, ld, rd)
    check_close(out, terms.sum(dim=1) + r.double(), err)
    assert torch.equal(out[::9], rd[::9])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer(xd, ld, rd)
    for i in range(4):
        ld.copy_(logits.roll(i, dims=1) + (i == 3) * 5.0 * (torch.arange(experts) < k))   # (the last: all tokens want the same experts)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, layer(xd, ld, rd)), i


@pytest.mark.parametrize("rows,width,hidden", cases.FEEDFORWARD)
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_feedforward_layer(rows, width, hidden, dtype):
    dtype = TYPES[dtype]
    g = torch.Generator().manual_seed(rows)
    (w1, s1), (w2, s2) = random_mx4(g, (2 * hidden, width), 116, 122), random_mx4(g, (width, hidden), 116, 122)
    gamma = 1.0 + 0.1 * torch.randn(width, generator=g)
    layer = FeedForwardMX4(gamma.cuda(), nm.nm_mx4_pack(w1.cuda(), s1.cuda(), width, gated=True), nm.nm_mx4_pack(w2.cuda(), s2.cuda(), hidden))
    x, r = rows_of(g, rows, width, dtype), rows_of(g, rows, width, dtype)
    say(f"FeedForwardMX4 {rows} rows, {width} x {hidden}, {dtype}")
    xd, rd = x.cuda(), r.cuda()
    q, s, stream = nm.nm_rmsnorm_mx4(xd, gamma.cuda(), rd)
    v = values_of(q, s, width)
    q, s = nm.nm_linear_mx4(q, s, layer.up, rounded=True)
    check_rounded(q, s, *product_ref(v, values_of(w1, s1, width), gated=True))
    check_close(layer(xd, rd), *product_ref(values_of(q, s, hidden), values_of(w2, s2, hidden), None, stream.cpu()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(xd, rd)
    for i in range(3):
        xd.copy_((x.float() * (1 + i)).to(dtype))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, layer(xd, rd))
