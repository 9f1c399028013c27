"""Scaled 8-bit tensors and the products on them in 64 bits, from their definition, on the CPU."""
import math

import numpy as np
import torch

# exponent bias, mantissa bits, largest value
FORMATS = {"e4m3": (7, 3, 448.0), "e5m2": (15, 2, 57344.0)}


def table(fmt):
    """Value of each of the 256 codes."""
    bias, bits, _ = FORMATS[fmt]
    top = (1 << (7 - bits)) - 1
    out = []
    for c in range(256):
        e, m = (c & 127) >> bits, c & ((1 << bits) - 1)
        v = math.ldexp(m, 1 - bias - bits) if e == 0 else math.ldexp((1 << bits) + m, e - bias - bits)
        if fmt == "e4m3" and (c & 127) == 127:
            v = math.nan
        if fmt == "e5m2" and e == top:
            v = math.nan if m else math.inf
        out.append(-v if c & 128 else v)
    return np.array(out)


def values(codes, scales, group, fmt):
    """float64 [T, K] of codes [T, K] and scales [groups, >= T] (uint8 tensors or arrays)."""
    codes, scales = np.asarray(torch.as_tensor(codes).cpu()), np.asarray(torch.as_tensor(scales).cpu())
    T, K = codes.shape
    f = np.ldexp(1.0, scales[:, :T].astype(np.int64) - 127).T
    return table(fmt)[codes] * f[:, np.arange(K) // group]


def exponent(most, fmt):
    """Smallest e >= -100 with most <= (largest value of the format) * 2^e."""
    largest = FORMATS[fmt][2]
    e = -100
    if most > 0:
        e = max(e, math.frexp(most / largest)[1] - 2)
        while most > largest * 2.0 ** e:
            e += 1
    return e


def encode(v, fmt):
    """Codes of float64 values, to nearest with ties to the even mantissa, by search in the table of the format's values."""
    t = table(fmt)
    largest = FORMATS[fmt][2]
    pos = np.array([c for c in range(128) if np.isfinite(t[c]) and t[c] <= largest])
    val = t[pos]
    a = np.abs(np.asarray(v, dtype=np.float64))
    hi = np.clip(np.searchsorted(val, np.where(np.isfinite(a), a, 0.0)), 0, len(val) - 1)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - val[lo], val[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (pos[lo] % 2 == 0)), lo, hi)
    code = pos[pick].astype(np.uint8)
    nan, inf = (0x7F, 0x7F) if fmt == "e4m3" else (0x7E, 0x7C)
    code = np.where(np.isnan(a), nan, np.where(np.isinf(a), inf, code)).astype(np.uint8)
    return np.where(np.signbit(v) & ~np.isnan(a), code | 128, code).astype(np.uint8)


MOST = 1.75 * 2.0 ** 127


def quantised(x, group, fmt):
    """(codes [T, K], scales [groups, T]) of float64 [T, K]."""
    x = np.asarray(x, dtype=np.float64)
    T, K = x.shape
    x = np.where(np.isfinite(x), np.clip(x, -MOST, MOST), x)
    n = -(-K // group)
    w = np.zeros((T, n * group))
    w[:, :K] = x
    w = w.reshape(T, n, group)
    most = np.abs(np.where(np.isfinite(w), w, 0.0)).max(2)
    e = exponents(most, fmt)
    codes = encode(np.ldexp(w, -e[:, :, None]), fmt).reshape(T, n * group)[:, :K]
    return codes, (e + 127).astype(np.uint8).T


def exponents(most, fmt):
    """exponent() of every value of an array: a candidate from the logarithm, put right by the definition's own comparison."""
    largest = FORMATS[fmt][2]
    e = np.full(most.shape, -100, dtype=np.int64)
    some = most > 0
    e[some] = np.maximum(np.floor(np.log2(most[some] / largest)).astype(np.int64) - 1, -100)
    for _ in range(4):
        e += most > np.ldexp(largest, e)
    return e


def same_codes(got, want, fmt):
    """Equal, a NaN's sign and mantissa apart."""
    t = table(fmt)
    return bool(np.all((got == want) | (np.isnan(t[got]) & np.isnan(t[want]))))


def act(name, z):
    z = torch.as_tensor(z, dtype=torch.float64)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    return torch.clamp_min(z, 0) if name == "relu" else z


def slope(name, z):
    z = torch.as_tensor(z, dtype=torch.float64)
    if name == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    if name == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return (z > 0).double() if name == "relu" else torch.ones_like(z)
