"""Plain forms of the 8-bit paged caches' rows, and the tolerance of attention in parts."""
import math

import torch

from tests import paged_ref as ref

E4M3 = torch.float8_e4m3fn
RANGE = {torch.bfloat16: (-120, 120), torch.float16: (-15, 8)}


def codes_of():
    """The 127 codes of e4m3 that are not negative, as 64-bit numbers in order."""
    return torch.arange(127, dtype=torch.uint8).view(E4M3).double()


def quantise(x):
    """(codes as uint8, exponents' bytes) of rows x [...][d] of a 16-bit type, in 64 bits from the definition: the
    smallest e with max|x| <= 448 2^e over the finite elements, each x 2^-e to the nearest code, ties to the even
    one, NaN for what is not finite."""
    lo, hi = RANGE[x.dtype]
    v = x.double().cpu()
    fine = torch.isfinite(v)
    a = torch.where(fine, v, 0.0).abs().amax(-1)
    bounds = 448 * torch.exp2(torch.arange(lo, hi + 1, dtype=torch.float64))
    n = torch.searchsorted(bounds, a).clamp(max=hi - lo)
    e = n + lo
    y = torch.where(fine, v, 0.0) * torch.exp2(-e.double())[..., None]
    m = torch.minimum(y.abs(), torch.where(e == hi, 240.0, 448.0)[..., None].double())
    c = codes_of()
    j = torch.searchsorted(c, m).clamp(1, 126)
    below, above = m - c[j - 1], c[j] - m
    j = torch.where((below < above) | ((below == above) & (j % 2 == 1)), j - 1, j)
    codes = j.to(torch.uint8) | (torch.signbit(v).to(torch.uint8) << 7)
    codes = torch.where(fine, codes, torch.tensor(0x7f, dtype=torch.uint8))
    return codes.to(x.device), (e + 127).to(torch.uint8).to(x.device)


def values(codes, scale):
    """[pages][page][H][d] values in 64 bits of float8 codes and bytes [pages][H][page]."""
    return codes.view(torch.uint8).view(E4M3).double() * torch.exp2(scale.transpose(1, 2).double() - 127)[..., None]


def check_attention(o, lse, r, dtype, parts=1, small_weights=0.0):
    """ref.check_attention with what a row in parts adds, and weights below what the kernel holds.

    Parts: each part's log-sum-exp is held in 32 bits in base 2, |.| <= 64, and is formed with lg2, both within
    2^-19; the difference of two of them moves a part's weight by a factor 1 + 2 ln 2 2^-19 < 1 + 2^-18, so an
    element by at most 2^-17 sum p|v|, which is added to the 2^-20 of the single pass.
    small_weights: what weights may be off by, absolutely, over the largest weight of the row, summed over its keys."""
    rr, rl, mass, eps = r
    u = ref.UNIT[dtype]
    small = 2.0 ** -20 if dtype is torch.bfloat16 else 2.0 ** -17
    if parts > 1:
        small += 2.0 ** -17
    top = mass.amax(-1, keepdim=True)
    tol = u * (rr.abs() + 1.01 * mass) * 1.02 + (2 * eps[..., None] + small) * (mass + top) + small_weights + 2.0 ** -24
    err = (o.double() - rr).abs()
    assert torch.isfinite(o.float()).all()
    assert (err <= tol).all(), f"out: worst error / tolerance {(err / tol).max().item():.3g}"
    if lse is not None:
        empty = torch.isinf(rl)
        assert torch.equal(empty, torch.isinf(lse)) and (lse[empty] < 0).all()
        le = (lse.double() - rl).abs()[~empty]
        lt = (eps + (2.0 ** -20 if parts == 1 else 2.0 ** -17) + 2.0 ** -22 * rl.abs())[~empty]
        assert (le <= lt).all(), f"lse: worst error / tolerance {(le / lt).max().item():.3g}"
