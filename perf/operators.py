"""The 8-bit feed-forward operators as cases that can be timed.

Four kinds of pass:

norm    `nm_rmsnorm_q8`: rows of x (with the residual stream added first) are root-mean-square normalised and
        rounded to 8 bits under one scale a row; then `nm_dequantize_q8`, so that what comes back is the values
        that the 8 bits stand for
quant   `nm_quantize_q8` and `nm_dequantize_q8`: the same rounding without a norm
linear  `nm_linear_q8`: 8-bit rows times 8-bit weights, a scale for each row and for each output channel, with a
        bias; or its gated form, silu(gate) * up of two products of the same rows
block   the operators as a transformer's feed-forward half uses them: residual addition and norm, gated product,
        rounding of its rows, second product with the residual stream added (`FeedForwardQ8`)

Sizes: the single tokens, decoding batches and prompts of a model with rows of 4096 and 8192; the classifier that
the benchmark's 50-layer network has (2048 to 1000, batch 64); and sizes off every tile.
"""
from __future__ import annotations

import torch

own = False

_DEV = "cuda:0"
_T = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_EPS = 1e-6
_MOST_FLOPS = 2.0 * 4096 * 4096 * 3 * 12288       # the largest listed case's products
_MOST_CELLS = 16384 * 8192                        # the largest listed case's elements in the row operators


def _case(name, c):
    return {"name": name, **c} if name else c


def _norm(name, rows, width, dtype, residual, gap=0):
    """gap: elements between the rows of x, as in a slice of a wider tensor."""
    return _case(name, {"kind": "norm", "rows": rows, "width": width, "dtype": dtype, "residual": residual, "gap": gap})


def _quant(name, rows, width, dtype, gap=0):
    return _case(name, {"kind": "quant", "rows": rows, "width": width, "dtype": dtype, "gap": gap})


def _linear(name, rows, k, n, dtype, bias=False, gated=False):
    """n: channels of the output (a gated product has 2 n rows of weights)."""
    return _case(name, {"kind": "linear", "rows": rows, "k": k, "n": n, "dtype": dtype, "bias": bias, "gated": gated})


def _block(name, rows, width, hidden):
    return _case(name, {"kind": "block", "rows": rows, "width": width, "hidden": hidden})


def listed():
    return [
        # one token of a decoding step: latency
        _norm("norm_1x4096_bf16", 1, 4096, "bf16", True),
        # fp32 rows of an odd width, none of them aligned, no residual stream
        _norm("norm_777x5001_f32", 777, 5001, "f32", False),
        # a long prompt's rows
        _norm("norm_16384x8192_bf16", 16384, 8192, "bf16", True),
        # a few rows of an odd width
        _quant("quant_65x1001_f32", 65, 1001, "f32"),
        # a prompt's hidden rows before the second product
        _quant("quant_8192x16384_bf16", 8192, 16384, "bf16"),
        # one token through a square layer: the weights are read once, latency counts
        _linear("linear_1x4096x4096_bf16", 1, 4096, 4096, "bf16"),
        # the classifier of the benchmark's network at its batch, logits in fp32
        _linear("linear_64x2048x1000_f32", 64, 2048, 1000, "f32", bias=True),
        # sizes off every tile, rows that start at odd addresses
        _linear("linear_333x1037x2501_bf16", 333, 1037, 2501, "bf16", bias=True),
        # the gated product of a short prompt
        _linear("gated_300x4096x8192_bf16", 300, 4096, 8192, "bf16", gated=True),
        # a long prompt through a wide layer
        _linear("linear_8192x4096x16384_bf16", 8192, 4096, 16384, "bf16"),
        # the feed-forward half of a decoding batch
        _block("block_16x4096x12288", 16, 4096, 12288),
        # the same of a prompt
        _block("block_4096x4096x12288", 4096, 4096, 12288),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm; two in five are multiples of 64 where that fits."""
    v = int(round(lo * (hi / lo) ** rng.random()))
    if rng.random() < 0.4 and v >= 64:
        v -= v % 64
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["norm", "quant", "linear", "linear", "gated", "block"])
    while True:
        if kind in ("norm", "quant"):
            rows, width, dtype = _spread(rng, 1, 16384), _spread(rng, 64, 16384), rng.choice(["bf16", "bf16", "f32"])
            gap = rng.choice([0, 0, 8, 3])
            if rows * width * _SIZE[dtype] <= _MOST_CELLS * 2:
                return _norm("", rows, width, dtype, rng.random() < 0.6, gap) if kind == "norm" else _quant("", rows, width, dtype, gap)
        elif kind == "block":
            rows, width, hidden = _spread(rng, 1, 4096), _spread(rng, 256, 8192), _spread(rng, 512, 16384)
            if 6.0 * rows * width * hidden <= _MOST_FLOPS and width * hidden <= 4096 * 12288:
                return _block("", rows, width, hidden)
        else:
            rows, k, n = _spread(rng, 1, 8192), _spread(rng, 64, 16384), _spread(rng, 64, 16384)
            gated = kind == "gated"
            if (4.0 if gated else 2.0) * rows * k * n <= _MOST_FLOPS and k * n <= 4096 * 16384:
                return _linear("", rows, k, n, rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.5, gated)


# ------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device=_DEV).manual_seed(int(seed))


def _rows(g, rows, width, dtype, gap, outliers=True):
    """Activations: normal, with a few channels that are much larger than the rest."""
    x = torch.randn((rows, width + gap), generator=g, device=_DEV)
    if outliers:
        x[:, :: max(1, width // 4)] *= 12.0
    return x.to(_T[dtype])[:, :width]


def _weights8(g, n, k):
    """Weights as a checkpoint in 8 bits has them: whole numbers in [-127, 127] and a scale for each channel."""
    w = (torch.randn((n, k), generator=g, device=_DEV) * 36.0).round_().clamp_(-127, 127).to(torch.int8)
    s = (0.5 + torch.rand(n, generator=g, device=_DEV)) / (36.0 * k ** 0.5)
    return w, s


def _handle(w, s, gated):
    from paper_2507_17301_amd import binding as nm
    return nm.nm_q8_pack(w, s, gated=gated)


def prepare(case, seed):
    g = _generator(seed)
    st = {"case": case}
    if case["kind"] in ("norm", "quant"):
        st["x"] = _rows(g, case["rows"], case["width"], case["dtype"], case["gap"])
        if case["kind"] == "norm":
            st["gamma"] = 1.0 + 0.1 * torch.randn(case["width"], generator=g, device=_DEV)
            st["residual"] = _rows(g, case["rows"], case["width"], case["dtype"], 0) if case["residual"] else None
    elif case["kind"] == "linear":
        wide = case["n"] * (2 if case["gated"] else 1)
        st["q"] = (torch.randn((case["rows"], case["k"]), generator=g, device=_DEV) * 32.0).round_().clamp_(-127, 127).to(torch.int8)
        st["s"] = (0.5 + torch.rand(case["rows"], generator=g, device=_DEV)) / 32.0
        st["w"], st["ws"] = _weights8(g, wide, case["k"])
        st["bias"] = 0.1 * torch.randn(wide, generator=g, device=_DEV) if case["bias"] else None
        if own:
            st["handle"] = _handle(st["w"], st["ws"], case["gated"])
    else:
        width, hidden = case["width"], case["hidden"]
        st["x"] = _rows(g, case["rows"], width, "bf16", 0, outliers=False)
        st["residual"] = _rows(g, case["rows"], width, "bf16", 0)
        st["gamma"] = 1.0 + 0.1 * torch.randn(width, generator=g, device=_DEV)
        st["w1"], st["ws1"] = _weights8(g, 2 * hidden, width)
        st["w2"], st["ws2"] = _weights8(g, width, hidden)
        if own:
            from paper_2507_17301_amd.feedforward import FeedForwardQ8
            st["layer"] = FeedForwardQ8(st["gamma"], _handle(st["w1"], st["ws1"], True), _handle(st["w2"], st["ws2"], False), eps=_EPS)
    return st


# ------------------------------------------------------------------ one pass
def _plain_round(v):
    """Rows of fp32 values as whole numbers (kept in fp32) and the scale of each row."""
    most = v.abs().amax(dim=1)
    scale = most / 127.0
    return torch.round(v * (127.0 / most)[:, None]).clamp(-127, 127), scale


def _plain_norm(x, residual, gamma):
    h = x.float() if residual is None else x.float() + residual.float()
    v = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + _EPS) * gamma
    q, s = _plain_round(v)
    return q, s, h


def _plain_product(q, s, w, ws, bias):
    y = (q.float() @ w.float().t()) * s[:, None] * ws
    return y if bias is None else y + bias


def _plain_gate(y):
    gate, up = y.chunk(2, dim=1)
    return gate / (1.0 + torch.exp(-gate)) * up


def _plain(st):
    case = st["case"]
    if case["kind"] == "norm":
        q, s, h = _plain_norm(st["x"], st["residual"], st["gamma"])
        out = {"values": (q * s[:, None]).to(torch.bfloat16), "scales": s}
        if st["residual"] is not None:
            out["stream"] = h.to(st["x"].dtype)
        return out
    if case["kind"] == "quant":
        q, s = _plain_round(st["x"].float())
        return {"values": (q * s[:, None]).to(torch.bfloat16), "scales": s}
    if case["kind"] == "linear":
        y = _plain_product(st["q"], st["s"], st["w"], st["ws"], st["bias"])
        return (_plain_gate(y) if case["gated"] else y).to(_T[case["dtype"]])
    q, s, h = _plain_norm(st["x"], st["residual"], st["gamma"])
    stream = h.to(torch.bfloat16)
    hidden = _plain_gate(_plain_product(q, s, st["w1"], st["ws1"], None)).to(torch.bfloat16)
    q, s = _plain_round(hidden.float())
    return (_plain_product(q, s, st["w2"], st["ws2"], None) + stream.float()).to(torch.bfloat16)


def run(st):
    if not own:
        return _plain(st)
    from paper_2507_17301_amd import binding as nm
    case = st["case"]
    if case["kind"] == "norm":
        q, s, stream = nm.nm_rmsnorm_q8(st["x"], st["gamma"], st["residual"], _EPS)
        out = {"values": nm.nm_dequantize_q8(q, s, torch.bfloat16), "scales": s}
        if stream is not None:
            out["stream"] = stream
        return out
    if case["kind"] == "quant":
        q, s = nm.nm_quantize_q8(st["x"])
        return {"values": nm.nm_dequantize_q8(q, s, torch.bfloat16), "scales": s}
    if case["kind"] == "linear":
        return nm.nm_linear_q8(st["q"], st["s"], st["handle"], st["bias"], dtype=_T[case["dtype"]])
    return st["layer"].forward(st["x"], st["residual"])


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] in ("norm", "quant"):
        cells, e = case["rows"] * case["width"], _SIZE[case["dtype"]]
        moved = e + 1 + 2                                    # x in, the 8 bits and the values they stand for out
        if case["kind"] == "norm":
            moved += 2 * e if case["residual"] else 0        # the stream in and out
        return {"bytes": cells * moved + 4 * case["rows"] + (4 * case["width"] if case["kind"] == "norm" else 0), "flops": 8 * cells}
    if case["kind"] == "linear":
        wide = case["n"] * (2 if case["gated"] else 1)
        return {"bytes": case["rows"] * (case["k"] + 4) + wide * (case["k"] + 4 + (4 if case["bias"] else 0)) + case["rows"] * case["n"] * _SIZE[case["dtype"]],
                "flops": 2.0 * case["rows"] * case["k"] * wide}
    width, hidden = case["width"], case["hidden"]
    return {"bytes": 3 * case["rows"] * width * 2 + 3 * width * hidden + 4 * (2 * width + 2 * hidden), "flops": 6.0 * case["rows"] * width * hidden}


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_scaled(v):
    """(whole numbers, scales) of rows in 64 bits."""
    scale = torch.linalg.vector_norm(v, ord=float("inf"), dim=1) / 127
    return (v / scale.unsqueeze(1)).round(), scale


def _exact_normed(st):
    h = st["x"].double()
    if st["residual"] is not None:
        h = h + st["residual"].double()
    return h, st["gamma"].double() * h / (h.pow(2).sum(1, keepdim=True) / h.shape[1] + _EPS).sqrt()


def _exact_linear(q, s, w, ws):
    """Sums of whole numbers: exact in 64 bits, since they stay under 2^53."""
    return torch.mm(q.double(), w.double().t()).mul_(s.double().unsqueeze(1)).mul_(ws.double())


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] in ("norm", "quant"):
        h, v = _exact_normed(st) if case["kind"] == "norm" else (None, st["x"].double())
        q, s = _exact_scaled(v)
        out = {"values": q * s.unsqueeze(1), "scales": s}
        if case["kind"] == "norm" and case["residual"]:
            out["stream"] = h
        return out
    if case["kind"] == "linear":
        y = _exact_linear(st["q"], st["s"], st["w"], st["ws"])
        if st["bias"] is not None:
            y = y + st["bias"].double()
        return y[:, : case["n"]] * torch.sigmoid(y[:, : case["n"]]) * y[:, case["n"]:] if case["gated"] else y
    h, v = _exact_normed(st)
    q, s = _exact_scaled(v)
    y = _exact_linear(q, s, st["w1"], st["ws1"])
    # the hidden rows and the stream are tensors in bf16: that rounding belongs to the operators' definition
    hidden = (y[:, : case["hidden"]] * torch.sigmoid(y[:, : case["hidden"]]) * y[:, case["hidden"]:]).to(torch.bfloat16).double()
    q, s = _exact_scaled(hidden)
    return _exact_linear(q, s, st["w2"], st["ws2"]) + h.to(torch.bfloat16).double()
