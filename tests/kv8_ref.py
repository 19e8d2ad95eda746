"""Plain references for normed heads and for the cache of 8-bit elements, in
float64: the elements by search among all of them, norms and rotary positions
with a bound on what the kernel may be off by."""
from __future__ import annotations

import torch

from kv_ref import UNIT, rotate

TOP = {"f32": 120, "f16": 8, "bf16": 120}  # 256 2^e is past the type's largest number


def element_values():
    """What the bytes 0 .. 126 stand for, from the format's definition: 4
    exponent bits with bias 7, 3 mantissa bits, subnormals below 2^-6."""
    out = []
    for b in range(127):
        e, m = b >> 3, b & 7
        out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return torch.tensor(out, dtype=torch.float64)


def scale_exponent(x):
    """Of each row [..., D] (float64, finite ones count): the least e >= -126
    with max |x| <= 448 2^e."""
    m = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    e = torch.full(m.shape, 130, dtype=torch.int32)
    for k in range(129, -127, -1):
        e = torch.where(m <= 448.0 * 2.0 ** k, torch.full_like(e, k), e)
    return e


def quantise(x, dtype):
    """(elements [..., D] uint8, scale bytes [...] uint8, the values they stand
    for) of rows x (float64 values of type dtype)."""
    e = scale_exponent(x)
    table = element_values()
    y = (x / torch.exp2(e.double())[..., None])
    a = y.abs()
    most = torch.where(e >= TOP[dtype], 240.0, 448.0)[..., None]
    a = torch.minimum(a, most.expand_as(a))
    hi = torch.searchsorted(table, a.nan_to_num(0.0).contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = a - table[lo], table[hi] - a
    pick = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)  # an even byte: an even mantissa
    byte = pick + 128 * torch.signbit(y).long()
    value = torch.copysign(table[pick], y) * torch.exp2(e.double())[..., None]
    bad = ~torch.isfinite(x)
    byte = torch.where(bad, torch.full_like(byte, 127), byte)
    value = torch.where(bad, torch.full_like(value, float("nan")), value)
    return byte.to(torch.uint8), (e + 127).to(torch.uint8), value


def page_bytes(byte, scale):
    """Elements [..., P, D] and scales [..., P] as a page's head [..., P D + P]."""
    return torch.cat((byte.flatten(-2), scale), dim=-1)


def split_page(raw, P, D):
    """(elements [..., P, D], scales [..., P]) of page heads [..., P D + P]."""
    return raw[..., :P * D].unflatten(-1, (P, D)), raw[..., P * D:]


def values_of(byte, scale):
    """What elements [..., P, D] under scales [..., P] stand for."""
    table = torch.cat((element_values(), torch.tensor([float("nan")], dtype=torch.float64)))
    v = table[(byte & 127).long()]
    return torch.where(byte > 127, -v, v) * torch.exp2(scale.double() - 127)[..., None]


def normed(x, weight, eps):
    x = x.double()
    mean = x.square().mean(-1, keepdim=True) + eps
    y = torch.where(mean > 0, x / mean.sqrt(), torch.zeros_like(x))
    return y if weight is None else y * weight.double()


def norm_rotate(x, weight, eps, cos, sin, pos, interleaved, dtype):
    """(exact, bound) of heads x [n][H][D] normed, turned and rounded once.  The
    kernel's relative error before the turn, in units of 2^-24: the sum of squares
    is of positive terms, at most 2 x 8 in a chain and 6 levels of lanes (23
    roundings), the division by D and eps 2, half of that from the root; the root 2,
    its reciprocal 2, two products 2, the weight 1: below 22.  The turn has two
    products and a sum (2 on each side): 24 of |a c| + |b s|; 28 are allowed, the
    factor covering second order."""
    y = x.double() if eps is None else normed(x, weight, eps)
    size = y.abs()
    if cos is not None:
        y = rotate(y, cos, sin, pos, interleaved)
        size = rotate_size(size, cos, sin, pos, interleaved)
    least = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -150}[dtype]
    return y, 28 * 2.0 ** -24 * size + UNIT[dtype] * y.abs() * (1 + 2.0 ** -18) + least


def rotate_size(a, cos, sin, pos, interleaved):
    """|a c| + |b s| of magnitudes a, pair by pair."""
    R = 2 * cos.shape[1]
    c, s = cos.double().abs()[pos][:, None], sin.double().abs()[pos][:, None]
    y = a.clone()
    i = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    p, q = a[..., i[0]], a[..., i[1]]
    y[..., i[0]], y[..., i[1]] = p * c + q * s, q * c + p * s
    return y
