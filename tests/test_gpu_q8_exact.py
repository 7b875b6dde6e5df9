"""Where the 8-bit operators have one right answer, or an error bound that the magnitudes of the values do not widen."""
import numpy as np
import pytest
import torch

from paper_2507_17301_amd import binding as nm
from gpu_util import say
from q8_util import check_rounded

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _every_pair():
    """Rows that hold every bf16 significand at every binade that does not round to 0, of both signs, under every largest magnitude:
    (values fp32 [128, n], x * 127 / a rounded to the nearest, ties to even, in whole numbers [128, n])."""
    m, j = np.meshgrid(np.arange(128, 256), np.arange(10), indexing="ij")
    m, j = m.reshape(-1), j.reshape(-1)                      # a value is m * 2^-j
    rows, want = [], []
    for a in range(128, 256):
        there = (m <= (a << j)) & ~((j == 0) & (m > a))
        num, den = 127 * m, a << j
        q = num // den
        twice = 2 * (num - q * den)
        q = q + ((twice > den) | ((twice == den) & (q % 2 == 1)))
        value, q = np.where(there, m * 2.0 ** -j, 0.0), np.where(there, q, 0)
        rows.append(np.concatenate([value, -value, [a]]))
        want.append(np.concatenate([q, -q, [127]]))
    return torch.from_numpy(np.array(rows, dtype=np.float32)), torch.from_numpy(np.array(want, dtype=np.int8))


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_rounding_of_bf16_values_is_to_the_nearest_ties_to_even(dtype):
    """a = 3, x = 1.5 is 63.5 and gives 64, although 127 / 3 is no fp32 number."""
    x, want = _every_pair()
    for power in (0, -100, 100):
        xs = (x * 2.0 ** power).to(TYPES[dtype])
        assert torch.equal(xs.double(), x.double() * 2.0 ** power)
        say(f"every pair of bf16 significands x 2^{power} as {dtype}")
        q, _ = nm.nm_quantize_q8(xs.cuda())
        off = (q.cpu() != want)
        assert not off.any(), f"{int(off.sum())} of {off.numel()}, first {xs[off][0]} in row {int(off.nonzero()[0, 0])}: {q.cpu()[off][0]} for {want[off][0]}"
        # channels of weights are rounded the same way
        assert np.array_equal(nm.nm_q8_export(nm.nm_q8_pack(xs.cuda()))[0], want.numpy())


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("width", [3, 300, 700, 1500, 4096, 5001, 20000])
def test_norm_of_rows_whose_squares_fp32_does_not_hold(width, dtype):
    """With no eps, or a tiny one, a norm does not depend on the magnitude of the row.  Bound: that of q8_util for the norm, 1e-5."""
    g = torch.Generator().manual_seed(width)
    x = torch.randn((12, width), generator=g)
    x[:, width // 2] = 5.0
    x *= torch.tensor([1e-8, 1e-11, 1e-13, 1e-18, 1e-20, 1e-21, 1e-22, 1e-23, 1e-26, 1e-30, 1e-34, 4e-36])[:, None]
    x = x.to(TYPES[dtype])
    gamma = 1 + 0.2 * torch.randn(width, generator=g)
    for eps in (0.0, 1e-44, 1e-40, 1e-24):
        e32 = float(np.float32(eps))
        for r in (None, x.flip(1).contiguous()):
            say(f"tiny rows of {width} {dtype} eps {eps} residual {r is not None}")
            q, s, _ = nm.nm_rmsnorm_q8(x.cuda(), gamma.cuda(), None if r is None else r.cuda(), eps)
            h = (x.float() if r is None else x.float() + r.float()).double().numpy()
            v = gamma.double().numpy() * h / np.sqrt((h ** 2).mean(axis=1, keepdims=True) + e32)
            check_rounded(q, s, v, 1e-5)
    # one that is zero, or whose root mean square is below 1.5e-36, has none; its neighbours are not touched
    x[1], x[4], x[7] = 0, 1e-38, 0
    q, s, _ = nm.nm_rmsnorm_q8(x.cuda(), gamma.cuda(), None, 0.0)
    h = x.double().numpy()
    for i in range(12):
        if i in (1, 4, 7):
            assert torch.isnan(s[i]) and not q[i].any()
        else:
            check_rounded(q[i:i + 1], s[i:i + 1], gamma.double().numpy() * h[i:i + 1] / np.sqrt((h[i:i + 1] ** 2).mean()), 1e-5)
    # with an eps above that, they are zero rows or tiny ones
    q, s, _ = nm.nm_rmsnorm_q8(x.cuda(), gamma.cuda(), None, 1e-30)
    assert s[1] == 0 and s[7] == 0 and not q[1].any() and not q[7].any() and torch.isfinite(s).all()


def test_rounding_of_fp32_values_next_to_half_steps():
    """Quotients x * 127 / a on both sides of every half step, and on it.  To the even number on it; to the nearest, except where the quotient
    rounded to fp32 lies on the half step, within half its spacing under 128: 2^-18."""
    rng = np.random.default_rng(3)
    a = np.concatenate([(1 + rng.random(60)).astype(np.float32), np.float32([1, 1.5, 127, 254, 3, 1.9999999, 1e-36 * 1.6, 3e38, 1e30])])
    near = ((np.arange(127) + 0.5) * a[:, None].astype(np.longdouble) / 127).astype(np.float32)     # [rows, 127]
    x = near
    for up in (np.float32(np.inf), np.float32(-np.inf)):
        y = near
        for _ in range(24):
            y = np.nextafter(y, up)
            x = np.concatenate([x, y], axis=1)
    x = np.concatenate([x, -x, rng.uniform(-1, 1, (len(a), 4000)).astype(np.float32) * a[:, None], a[:, None]], axis=1)
    x = np.where(np.abs(x) <= a[:, None], x, np.float32(0))
    v = np.abs(x.astype(np.longdouble)) * 127 / a[:, None].astype(np.longdouble)
    low = np.floor(v)
    tie = 2 * 127 * np.abs(x.astype(np.longdouble)) == (2 * low + 1) * a[:, None].astype(np.longdouble)     # (exact: 32 bits)
    assert tie.sum() > 300
    nearest = np.where(tie, low + low % 2, np.rint(v))
    say(f"fp32 values next to half steps, {x.shape}")
    q, _ = nm.nm_quantize_q8(torch.from_numpy(x).cuda())
    q = q.cpu().numpy().astype(np.int32)
    assert (q * np.sign(x) >= 0).all()
    off = (np.abs(q) != nearest) & (tie | (np.abs(v - low - 0.5) > 2.0 ** -18)) | (np.abs(np.abs(q) - nearest) > 1)
    assert not off.any(), f"{off.sum()} of {off.size}, first {x[off][0]!r} in a row of {a[np.argwhere(off)[0, 0]]!r}: {q[off][0]}"
