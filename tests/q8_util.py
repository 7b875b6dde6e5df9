"""References in 64 bits for the 8-bit operators, and the bounds that their results are held to.

Bounds follow from the formulas, with u = 2^-24 (one rounding to fp32):
  scales of nm_quantize_q8   one division of exact values: equal to fp32 division bit for bit
  q                          |q - x * 127 / a| <= 1/2 + 127 * (relative error of x * 127 / a before the rounding), which is
                             3 u for nm_quantize_q8 and, for the norm, that of v / max|v|
  norm                       a sum of n squares in fp32, at most 64 in a row and then a tree: relative error under
                             (64 + 16) u, halved by the square root; with the products, under 1e-5
  product                    the integer sum is exact; three roundings of the scaled sum, one of each addition
  gated                      exp() in fp32 of an argument with relative error 2 u: relative error (2 |z| + 4) u
  bf16 outputs               one more rounding of relative size 2^-9 (and half the smallest subnormal)
"""
import numpy as np
import torch

U = 2.0 ** -24


def rows_of(gen, rows, width, dtype, gap=0, scale=1.0):
    x = torch.randn((rows, width + gap), generator=gen) * scale
    x[:, :: max(1, width // 3)] *= 9.0
    return x.to(dtype)


def on_gpu(x, width):
    """The first `width` columns of a (wider) tensor, on the device, as a view of the wide one."""
    return x.cuda()[:, :width]


def check_rounded(q, s, v, rel):
    """q, s (tensors) against the rows v (64 bits) that they round, known up to the relative error `rel` of a row's values."""
    q, s, v = q.cpu().double().numpy(), s.cpu().double().numpy().reshape(-1), np.asarray(v, dtype=np.float64)
    q = q.reshape(v.shape)
    a = np.abs(v).max(axis=1)
    assert np.all(np.abs(s - a / 127) <= (rel + 2 * U) * a / 127)
    with np.errstate(divide="ignore", invalid="ignore"):
        want = np.where(a[:, None] > 0, v * (127 / a)[:, None], 0.0)
    off = np.abs(q - want)
    assert off.max() <= 0.5 + 127 * (2 * rel + 4 * U), off.max()
    assert np.abs(q).max(initial=0) <= 127


def linear_ref(q, s, w, ws, bias=None, residual=None, gated=False):
    """(result, bound of the error in fp32) in 64 bits, on the CPU."""
    q, s, w, ws = (t.cpu().double() for t in (q, s, w, ws))
    a = (q @ w.t()) * s[:, None] * ws
    z = a if bias is None else a + bias.cpu().double()
    e = 4 * U * (a.abs() + (0 if bias is None else bias.cpu().double().abs()))
    if gated:
        half = z.shape[1] // 2
        g, v, eg, ev = z[:, :half], z[:, half:], e[:, :half], e[:, half:]
        sig = torch.sigmoid(g)
        y = g * sig * v
        # |d silu / d g| <= 1.1; the errors of exp, the sum, the quotient and the product
        return y, 1.1 * eg * v.abs() + (g * sig).abs() * ev + y.abs() * (2 * g.abs() + 8) * U + 1e-37
    if residual is not None:
        r = residual.cpu().double()
        z, e = z + r, e + 2 * U * (z.abs() + r.abs())
    return z, e


def check_close(y, ref, bound):
    y64 = y.cpu().double()
    if y.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (ref.abs() + bound) + 2.0 ** -133
    off = (y64 - ref).abs() - bound
    assert torch.isfinite(y64).all()
    assert off.max() <= 0, f"worst excess {off.max():.3g} at {np.unravel_index(int(off.argmax()), off.shape)}"
