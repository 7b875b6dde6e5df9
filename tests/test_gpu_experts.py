"""Routing, products grouped by expert, their combination and the layer of experts against their formulas in 64 bits."""
import math

import pytest
import torch

from paper_2507_17301_amd import binding as nm
from paper_2507_17301_amd.feedforward import ExpertsMX4
from gpu_util import say
from mx4_util import U, blocks, check_close, check_rounded, product_ref, random_mx4, round_ref, rows_of, values_of

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ routing
def route_ref(logits, k, normalise=True):
    """Choices one after another; the order by counting."""
    tokens, experts = logits.shape
    key = torch.where(torch.isnan(logits), torch.full_like(logits, math.inf), logits).double()
    nan = torch.isnan(logits)
    # NaN first, then by value, ties by expert: sorted stably by the last criterion first
    order = torch.argsort(-key, dim=1, stable=True)
    order = torch.gather(order, 1, torch.argsort((~torch.gather(nan, 1, order)).int(), dim=1, stable=True))
    ids = order[:, :k].clone()
    best = torch.gather(logits.double(), 1, ids)
    closed = best == -math.inf
    ids[closed] = -1
    e = torch.where(closed, 0.0, torch.exp(best - best[:, :1]))
    total = e.sum(dim=1, keepdim=True) if normalise else torch.exp(logits.double() - best[:, :1]).sum(dim=1, keepdim=True)
    weights = torch.where(closed, 0.0, e / total)
    rows, slots, offsets = [], torch.full((tokens, k), -1, dtype=torch.int64), [0]
    for x in range(experts):
        for t, j in (ids == x).nonzero().tolist():
            slots[t, j] = len(rows)
            rows.append(t)
        offsets.append(len(rows))
    rows += [-1] * (tokens * k - len(rows))
    return ids, weights, offsets, rows, slots


def check_route(logits, k, normalise=True, ld=0):
    tokens, experts = logits.shape
    say(f"route {tokens} x {experts} k {k} {logits.dtype} normalise {normalise}")
    x = logits.cuda()
    if ld:
        wide = torch.full((tokens, experts + ld), 1e9, dtype=logits.dtype, device="cuda")
        wide[:, 1:1 + experts] = x
        x = wide[:, 1:1 + experts]
    got = nm.nm_route(x, k, normalise)
    ids, weights, offsets, rows, slots = route_ref(logits, k, normalise)
    assert torch.equal(got.ids.cpu().long(), ids) and got.offsets.tolist() == offsets
    assert got.rows.tolist() == rows and torch.equal(got.slots.cpu().long(), slots)
    w = got.weights.cpu().double()
    assert torch.equal(torch.isnan(w), torch.isnan(weights))
    # exp in fp32: its own 2 u and the argument's rounding, |l| u at most; the sum of up to `experts` terms; the quotient
    spread = torch.where(torch.isfinite(logits.double()), logits.double().abs(), 0.0).amax() * 2
    bound = weights * ((2 * spread + 8 + experts) * U) + 1e-37
    assert torch.nan_to_num((w - weights).abs() - bound, nan=0.0).max() <= 0
    return got


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("experts", [1, 2, 15, 16, 17, 63, 64, 65, 200, 256, 257, 512, 1000, 1024])
def test_routing(experts, dtype):
    g = torch.Generator().manual_seed(experts)
    for i, tokens in enumerate((1, 2, 63, 64, 65, 130, 700)):
        if tokens == 700 and experts > 300:
            continue
        k = min(experts, (1, 8, 3, 2, 64, 5, 4)[i])
        x = torch.randn((tokens, experts), generator=g)
        x = (x * 4).round() / 4 if i % 2 else x          # many ties
        check_route(x.to(TYPES[dtype]), k, i % 3 != 0, ld=i % 2 * 3)


def test_more_chunks_of_tokens_than_workgroups_hold_batches():
    g = torch.Generator().manual_seed(1)
    x = torch.randn((256 * 64 + 300, 8), generator=g)    # chunks of two batches
    got = nm.nm_route(x.cuda(), 2)
    best = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :2]
    flat = best.flatten()
    by = torch.sort(flat, stable=True)[1]
    assert torch.equal(got.ids.cpu().long(), best) and torch.equal(got.rows.cpu().long(), by // 2)
    assert got.offsets.tolist() == [int((flat < e).sum()) for e in range(9)]
    slots = torch.empty_like(by)
    slots[by] = torch.arange(by.numel())
    assert torch.equal(got.slots.cpu().long().flatten(), slots)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_closed_experts_padding_and_values_that_are_not_finite(dtype):
    g = torch.Generator().manual_seed(2)
    for tokens, experts, k in ((40, 20, 6), (300, 70, 8), (90, 300, 4)):
        x = torch.randn((tokens, experts), generator=g).to(TYPES[dtype])
        x.masked_fill_(torch.rand((tokens, experts), generator=g) < 0.8, -math.inf)
        x[::7] = -math.inf                               # padding
        x[3, 2], x[5, 4], x[5, 9], x[8, 1] = math.nan, math.nan, math.nan, math.inf
        x[9] = torch.finfo(TYPES[dtype]).min             # the type's lowest value is a number
        x[10, :] = -math.inf
        x[10, experts - 1] = -3.0                        # one open expert
        x[11, 0], x[11, 1], x[11, 2:] = 0.0, -0.0, -1.0  # equal
        got = check_route(x, k)
        assert (got.slots[::7] == -1).all() and (got.weights[::7] == 0).all()
        assert got.weights[10, 0] == 1 and torch.isnan(got.weights[3, 0]) and got.ids[3, 0] == 2
        assert got.ids[11, :2].tolist() == [0, 1]
    nothing = torch.full((50, 12), -math.inf, dtype=TYPES[dtype])
    got = check_route(nothing, 3)
    assert got.offsets.tolist() == [0] * 13 and (got.rows == -1).all()


def test_no_tokens_and_more_axes():
    got = nm.nm_route(torch.zeros((0, 9), device="cuda"), 2)
    assert got.offsets.tolist() == [0] * 10 and got.ids.shape == (0, 2) and got.rows.shape == (0,)
    x = torch.randn((4, 5, 33), device="cuda")
    a, b = nm.nm_route(x, 3), nm.nm_route(x.view(20, 33), 3)
    assert a.ids.shape == (4, 5, 3) and all(torch.equal(u.flatten(), v.flatten()) for u, v in zip(a, b))


# ------------------------------------------------------------------ combination
@pytest.mark.parametrize("ydt", sorted(TYPES))
@pytest.mark.parametrize("dt", sorted(TYPES))
def test_combination(dt, ydt):
    g = torch.Generator().manual_seed(5)
    for tokens, k, width, entries in ((1, 1, 1, 1), (3, 2, 7, 6), (20, 8, 64, 100), (50, 5, 1001, 260), (7, 64, 130, 30)):
        y = torch.randn((entries, width + 5), generator=g).to(TYPES[ydt])
        slots = torch.randint(-1, entries, (tokens, k), generator=g, dtype=torch.int32)
        weights = torch.rand((tokens, k), generator=g)
        r = torch.randn((tokens, width), generator=g).to(TYPES[dt]) if tokens != 3 else None
        say(f"combine {tokens} x {k} x {width} {dt} {ydt}")
        out = nm.nm_combine(y.cuda()[:, 2:2 + width], slots.cuda(), weights.cuda(), None if r is None else r.cuda(), TYPES[dt])
        terms = torch.where((slots >= 0)[..., None], weights.double()[..., None] * y.double()[slots.clamp(min=0).long()][..., 2:2 + width], 0.0)
        ref, size = terms.sum(dim=1), terms.abs().sum(dim=1)
        if r is not None:
            ref, size = ref + r.double(), size + r.double().abs()
        check_close(out, ref, (k + 2) * U * size)       # each product and sum rounds once
        if r is not None:
            rd = r.cuda()
            assert nm.nm_combine(y.cuda()[:, 2:2 + width], slots.cuda(), weights.cuda(), rd, out=rd) is rd and torch.equal(rd, out)
    y, w = torch.randn((4, 40), device="cuda"), torch.ones((3, 2), device="cuda")
    out = nm.nm_combine(y, torch.tensor([[0, 1], [2, 4], [-2, 3]], dtype=torch.int32, device="cuda"), w)
    assert torch.equal(out[0], y[0] + y[1]) and torch.isnan(out[1]).all() and torch.isnan(out[2]).all()
    assert (nm.nm_combine(y[:0], torch.full((3, 2), -1, dtype=torch.int32, device="cuda"), w) == 0).all()


# ------------------------------------------------------------------ grouped products
def groups_of(g, experts, entries, kind):
    """Sizes of groups that add up to `entries`."""
    if kind == "one":
        n = [0] * experts
        n[experts // 2] = entries
    elif kind == "even":
        n = [entries // experts + (e < entries % experts) for e in range(experts)]
    else:                                               # ragged, some empty
        p = torch.rand(experts, generator=g) ** 4 * (torch.rand(experts, generator=g) < 0.7)
        n = torch.bincount(torch.multinomial(p + 1e-9, entries, True, generator=g), minlength=experts).tolist() if entries else [0] * experts
    return torch.tensor([0] + n).cumsum(0).int()


def grouped_ref(x, offsets, w, bias, gated):
    y, bound = [], []
    for e in range(len(offsets) - 1):
        part = product_ref(x[offsets[e]:offsets[e + 1]], w[e], None if bias is None else bias[e], None, gated)
        y.append(part[0])
        bound.append(part[1])
    return torch.cat(y), torch.cat(bound)


CASES = [(1, 1, 32, 4, "even"), (1, 5, 100, 33, "even"), (3, 7, 64, 64, "ragged"), (8, 40, 300, 70, "ragged"), (70, 100, 257, 40, "ragged"),
         (5, 130, 512, 130, "one"), (4, 300, 256, 200, "ragged"), (130, 900, 96, 65, "ragged"), (6, 1500, 300, 260, "ragged"), (3, 2100, 640, 300, "one"),
         (16, 2000, 200, 515, "even"), (64, 64, 1037, 30, "even")]


@pytest.mark.parametrize("out", ["bf16", "f32", "mx4"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("experts,entries,k,n,kind", CASES)
def test_grouped_products(experts, entries, k, n, kind, gated, out):
    g = torch.Generator().manual_seed(experts + entries)
    n = 2 * n if gated else n
    offsets = groups_of(g, experts, entries, kind)
    w, ws = random_mx4(g, (experts, n, k), 110, 122)
    bias = torch.randn((experts, n), generator=g) if entries % 2 == 0 else None
    h = nm.nm_mx4_pack(w.cuda(), ws.cuda(), k, gated=gated)
    wv, t = values_of(w, ws, k), TYPES.get(out)
    for tokens in (None, max(1, entries // 3)):
        q, s = random_mx4(g, (tokens or entries, k))
        index = torch.randint(0, tokens, (entries,), generator=g, dtype=torch.int32) if tokens else None
        say(f"experts_mx4 {experts} x {entries} x {k} x {n} {kind} gated {gated} {out} gather {tokens}")
        y = nm.nm_experts_mx4(q.cuda(), s.cuda(), h, offsets.cuda(), None if index is None else index.cuda(), None if bias is None else bias.cuda(), t,
                              rounded=t is None)
        torch.cuda.synchronize()
        x = values_of(q, s, k)
        ref = grouped_ref(x if index is None else x[index.long()], offsets, wv, bias, gated)
        if t is None:
            check_rounded(y[0], y[1], *ref)
        else:
            check_close(y, *ref)


@pytest.mark.parametrize("entries", [30, 400, 3000])
def test_rows_in_no_group_are_left_as_they_were(entries):
    g = torch.Generator().manual_seed(entries)
    experts, k, n = 5, 128, 100
    h = nm.nm_mx4_pack(*(v.cuda() for v in random_mx4(g, (experts, n, k), 110, 122)))
    q, s = (v.cuda() for v in random_mx4(g, (entries, k)))
    offsets = groups_of(g, experts, entries * 2 // 3, "ragged").cuda()
    end = int(offsets[-1])
    full = nm.nm_experts_mx4(q, s, h, offsets, dtype=torch.float32)
    y = torch.full((entries, n + 6), 5.0, device="cuda")
    nm.nm_experts_mx4(q, s, h, offsets, y=y[:, 2:2 + n])
    assert torch.equal(y[:end, 2:2 + n], full[:end]) and (y[end:] == 5).all() and (y[:, :2] == 5).all() and (y[:, 2 + n:] == 5).all()
    yq, ys = torch.full((entries, 64), 0x33, dtype=torch.uint8, device="cuda"), torch.full((entries, 4), 0x33, dtype=torch.uint8, device="cuda")
    nm.nm_experts_mx4(q, s, h, offsets, y=yq, y_scales=ys, rounded=True)
    assert (yq[end:] == 0x33).all() and (ys[end:] == 0x33).all() and not (ys[:end] == 0x33).all()
    none = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    y = torch.full((entries, n), 5.0, device="cuda")
    assert (nm.nm_experts_mx4(q, s, h, none, y=y) == 5).all()


@pytest.mark.parametrize("entries", [40, 700])
def test_offsets_and_rows_out_of_range(entries):
    """Offsets past the ends count as the ends, a falling one as an empty group; a row that there is not gives NaN."""
    g = torch.Generator().manual_seed(entries)
    experts, k, n = 4, 96, 70
    h = nm.nm_mx4_pack(*(v.cuda() for v in random_mx4(g, (experts, n, k), 110, 122)))
    q, s = (v.cuda() for v in random_mx4(g, (entries, k)))
    half = entries // 2
    good = nm.nm_experts_mx4(q, s, h, torch.tensor([0, half, half, half, entries], dtype=torch.int32, device="cuda"), dtype=torch.float32)
    bad = nm.nm_experts_mx4(q, s, h, torch.tensor([-7, half, half - 3, half, entries + 1000], dtype=torch.int32, device="cuda"),
                            dtype=torch.float32, y=torch.zeros((entries, n), device="cuda"))
    # (the third group, half - 3 .. half, is expert 2's as well: those three rows belong to two groups)
    keep = torch.ones(entries, dtype=torch.bool)
    keep[half - 3:half] = False
    assert torch.equal(bad[keep], good[keep])
    index = torch.arange(entries, dtype=torch.int32)
    index[5], index[entries - 1], index[9] = -1, entries, 2 ** 31 - 1
    off = torch.tensor([0, half, half, half, entries], dtype=torch.int32, device="cuda")
    y = nm.nm_experts_mx4(q, s, h, off, index.cuda(), dtype=torch.float32)
    lost = torch.zeros(entries, dtype=torch.bool)
    lost[5] = lost[9] = lost[entries - 1] = True
    assert torch.isnan(y[lost]).all() and torch.equal(y[~lost], good[~lost])
    _, ys = nm.nm_experts_mx4(q, s, h, off, index.cuda(), rounded=True)
    assert (ys[lost] == 255).all() and (ys[~lost] != 255).all()


def test_refusals():
    g = torch.Generator().manual_seed(1)
    h = nm.nm_mx4_pack(*(v.cuda() for v in random_mx4(g, (3, 20, 64), 110, 122)))
    q, s = (v.cuda() for v in random_mx4(g, (8, 64)))
    off = torch.tensor([0, 2, 5, 8], dtype=torch.int32, device="cuda")
    for call in (lambda: nm.nm_experts_mx4(q, s, h, None), lambda: nm.nm_experts_mx4(q, s, h, off[:3]), lambda: nm.nm_experts_mx4(q, s, h, off.long()),
                 lambda: nm.nm_experts_mx4(q, s, h, off, bias=torch.zeros(20, device="cuda")), lambda: nm.nm_experts_mx4(q, s, h, off.cpu()),
                 lambda: nm.nm_combine(torch.zeros((4, 8), device="cuda"), torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros((2, 1), device="cuda"))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(nm.NMError) as e:
        nm.nm_experts_mx4(q[:0], s[:0], h, off, torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert e.value.code == nm.NM_ERR_ARG
    for k, experts, code in ((0, 5, nm.NM_ERR_ARG), (6, 5, nm.NM_ERR_ARG), (65, 100, nm.NM_ERR_SHAPE), (2, 1025, nm.NM_ERR_SHAPE)):
        with pytest.raises(nm.NMError) as e:
            nm.nm_route(torch.zeros((3, experts), device="cuda"), k)
        assert e.value.code in (code, nm.NM_ERR_ARG)


# ------------------------------------------------------------------ the layer
def test_layer_and_graph():
    g = torch.Generator().manual_seed(31)
    experts, k, width, hidden = 9, 3, 160, 224
    gate, up = (torch.randn((experts, hidden, width), generator=g) / width ** 0.5 for _ in range(2))
    down = torch.randn((experts, width, hidden), generator=g) / hidden ** 0.5
    layer = ExpertsMX4.from_float(gate.cuda(), up.cuda(), down.cuda(), k)
    w1 = torch.stack([round_ref(torch.cat([gate[e], up[e]]))[0] for e in range(experts)])
    w2 = torch.stack([round_ref(down[e])[0] for e in range(experts)])
    for dtype in TYPES.values():
        for tokens in (1, 30, 500):
            x, r = rows_of(g, tokens, width, dtype), rows_of(g, tokens, width, dtype)
            logits = torch.randn((tokens, experts), generator=g)
            logits[::5] = -math.inf                      # padding: the residual stream comes back
            if tokens == 1:
                logits[:] = torch.randn(experts, generator=g)
            say(f"ExpertsMX4 {tokens} tokens {dtype}")
            ids, weights, offsets, rows, slots = route_ref(logits, k)
            n = offsets[-1]
            to = nm.nm_route(logits.cuda(), k)
            q, s = nm.nm_experts_mx4(*nm.nm_quantize_mx4(x.cuda()), layer.up, to.offsets, to.rows, rounded=True)
            check_rounded(q[:n], s[:n], *grouped_ref(round_ref(x.double())[0][rows[:n]], offsets, w1, None, True))
            # what the second product gets is the kernel's own rounding, held to its bound
            y, bound = grouped_ref(values_of(q[:n], s[:n], hidden), offsets, w2, None, False)
            if dtype == torch.bfloat16:
                bound = bound + 2.0 ** -8 * (y.abs() + bound)
            pick = torch.where(slots >= 0, slots, 0)
            open_ = (slots >= 0)[..., None]
            ref = torch.where(open_, weights[..., None] * y[pick], 0.0).sum(dim=1) + r.double()
            size = torch.where(open_, weights[..., None] * y[pick].abs(), 0.0).sum(dim=1) + r.double().abs()
            err = torch.where(open_, weights[..., None] * bound[pick], 0.0).sum(dim=1) + 40 * U * size
            out = layer(x.cuda(), logits.cuda(), r.cuda())
            check_close(out, ref, err)
            if tokens > 1:
                assert torch.equal(out[::5].cpu(), r[::5])
            xd, ld, rd = x.cuda(), logits.cuda(), r.cuda()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                got = layer(xd, ld, rd)
            for i in range(3):
                ld.copy_(logits.roll(i, dims=1))
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(got, layer(xd, ld, rd))
