"""References in 64 bits for the operators in MX4, and the bounds that their results are held to.

Bounds follow from the formulas, with u = 2^-24 (one rounding to fp32; at most 2 u where a sum is cut off instead):
  codes and scales   those of the formula, exactly: of given values no other rounding comes in; of a norm's, h and the two
                     products are single operations in fp32, and n is a 64-bit number rounded once
  product            products of two 4-bit values and two powers of two are exact.  An instruction adds 128 of them, the
                     accumulator K / 128 such sums, a workgroup's wavefronts or K's parts up to 32 of those: in any order an
                     error of at most (128 + K / 128 + 32) * 2 u * sum |p|; then one rounding for the bias and one for a residual
  gated              |d silu / d g| <= 1.1; exp() in fp32 of an argument with relative error 2 u: relative error (2 |g| + 8) u
  bf16 outputs       one more rounding of relative size 2^-8 (and half the smallest subnormal)
  outputs in MX4     the rounding of some number within the product's bound
"""
import numpy as np
import torch

U = 2.0 ** -24
LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
BORDERS = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]


def blocks(width):
    return (width + 31) // 32


def rows_of(gen, rows, width, dtype, gap=0, scale=1.0):
    x = torch.randn((rows, width + gap), generator=gen) * scale
    x[:, :: max(1, width // 3)] *= 9.0
    return x.to(dtype)


def on_gpu(x, width, at=0):
    """`width` columns of a (wider) tensor, on the device, as a view of the wide one."""
    return x.cuda()[:, at:at + width]


def scale_ref(a):
    """Scale bytes of blocks with the largest magnitudes a (64 bits)."""
    ok = torch.isfinite(a)
    e = torch.frexp(torch.where(ok, a, torch.ones_like(a)))[1] - 3          # floor(log2 a) - 2
    e = torch.where(a > 0, e, torch.full_like(e, -127)).clamp(min=-127)
    return torch.where(ok, e + 127, torch.full_like(e, 255)).to(torch.int64)


def level_ref(m):
    """Magnitudes in units of the block's power of two, rounded to a value of the type."""
    code = torch.zeros(m.shape, dtype=torch.int64)
    for i, b in enumerate(BORDERS):
        code += (m > b) if i % 2 == 0 else (m >= b)
    return LEVELS[code]


def round_ref(v):
    """(values [rows, width], scale bytes [rows, blocks]) of rows v in 64 bits; the values of NaN blocks are NaN."""
    v = torch.as_tensor(v, dtype=torch.float64)
    rows, width = v.shape
    full = torch.zeros((rows, blocks(width) * 32), dtype=torch.float64)
    full[:, :width] = v
    full = full.view(rows, -1, 32)
    a = full.abs().amax(dim=2)
    a = torch.where(torch.isfinite(full).all(dim=2), a, torch.full_like(a, float("inf")))
    s = scale_ref(a)
    p = torch.where(s == 255, torch.nan, 2.0 ** (s.double() - 127))[:, :, None]
    m = torch.nan_to_num(full.abs() / torch.nan_to_num(p, nan=1.0), nan=0.0, posinf=0.0)
    return (torch.copysign(level_ref(m), full) * p).reshape(rows, -1)[:, :width], s


def values_of(q, s, width):
    """The values in 64 bits that codes [.., 16 B] and scale bytes [.., B] stand for."""
    q, s = q.cpu().to(torch.int64), s.cpu().to(torch.int64)
    codes = torch.stack([q & 15, q >> 4], dim=-1).flatten(-2)
    size = LEVELS[codes & 7]
    p = torch.where(s == 255, torch.nan, 2.0 ** (s.double() - 127))
    v = torch.where(codes > 7, -size, size).unflatten(-1, (-1, 32)) * p[..., None]
    return v.flatten(-2)[..., :width]


def same(a, b):
    """Equal values, NaN to NaN, 0 to -0."""
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a, nan=0.0) + 0.0, torch.nan_to_num(b, nan=0.0) + 0.0)


def random_mx4(gen, shape, low=118, high=132):
    """(codes, scales) of any codes, and of powers of two around 1."""
    width, lead = shape[-1], shape[:-1]
    q = torch.randint(0, 256, lead + (blocks(width) * 16,), generator=gen, dtype=torch.uint8)
    return q, torch.randint(low, high, lead + (blocks(width),), generator=gen, dtype=torch.uint8)


def product_ref(x, w, bias=None, residual=None, gated=False):
    """(result, bound of the error in fp32) of rows x and weights w in 64 bits."""
    k = x.shape[1]
    z = x @ w.t()
    e = (128 + k / 128 + 32) * 2 * U * (x.abs() @ w.abs().t())
    if bias is not None:
        z = z + bias.double()
        e = e + 2 * U * (z.abs() + bias.double().abs())
    if gated:
        half = z.shape[1] // 2
        g, v, eg, ev = z[:, :half], z[:, half:], e[:, :half], e[:, half:]
        sig = torch.sigmoid(g)
        y = g * sig * v
        return y, 1.1 * eg * v.abs() + (g * sig).abs() * ev + 1.1 * eg * ev + y.abs() * (2 * g.abs() + 8) * U + 1e-37
    if residual is not None:
        r = residual.double()
        z = z + r
        e = e + 2 * U * (z.abs() + r.abs())
    return z, e


def check_close(y, ref, bound):
    y64 = y.cpu().double()
    if y.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (ref.abs() + bound) + 2.0 ** -133
    off = (y64 - ref).abs() - bound
    assert torch.isfinite(y64).all()
    assert off.numel() == 0 or off.max() <= 0, f"worst excess {off.max():.3g} at {np.unravel_index(int(off.argmax()), off.shape)}"


def check_rounded(q, s, ref, bound):
    """Codes and scales against rows that are known up to `bound`."""
    rows, width = ref.shape
    n = blocks(width)
    assert q.shape == (rows, n * 16) and s.shape == (rows, n)
    pad = torch.zeros((rows, n * 32), dtype=torch.float64)
    pad[:, :width] = ref
    err = torch.zeros_like(pad)
    err[:, :width] = bound
    a, e = pad.abs().view(rows, n, 32), err.view(rows, n, 32)
    low, high = (a - e).clamp(min=0).amax(dim=2), (a + e).amax(dim=2)
    got = s.cpu().to(torch.int64)
    assert (got >= scale_ref(low)).all() and (got <= scale_ref(high)).all()
    p = (2.0 ** (got.double() - 127))[:, :, None]
    v = values_of(q, s, n * 32).view(rows, n, 32) / p
    def level(x):
        return torch.copysign(level_ref(x.abs()), x)
    x = pad.view(rows, n, 32)
    assert (v >= level((x - e) / p)).all() and (v <= level((x + e) / p)).all()
