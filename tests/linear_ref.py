"""The linear layer's operators in 64 bits, from their definitions: the
8-bit checkpoints by nearest value in a table of the format's codes, the
products and activations in float64.  No code of the package is used."""
from __future__ import annotations

import math

import torch

ROWS, COLS, MAX_FT = 32, 128, 96
FORMATS = {"1-5-2": (5, 2, 15), "1-4-3": (4, 3, 7)}
EMAX = {torch.float32: 127, torch.bfloat16: 127, torch.float16: 15}


def table(fmt: str) -> torch.Tensor:
    """The values of the 256 codes, float64."""
    e, m, bias = FORMATS[fmt]
    v = []
    for c in range(256):
        field, mant = (c & 127) >> m, c & ((1 << m) - 1)
        if field == (1 << e) - 1:
            a = math.nan if mant else math.inf
        else:
            a = math.ldexp(mant + ((1 << m) if field else 0), max(field, 1) - bias - m)
        v.append(-a if c & 128 else a)
    return torch.tensor(v, dtype=torch.float64)


def limit(fmt: str, T) -> float:
    return math.ldexp(2 - 2.0 ** -FORMATS[fmt][1], EMAX[T])


def _ceil_log2(x: float) -> int:
    f, e = math.frexp(x)
    return e - 1 if f == 0.5 else e


def block_exponents(x: torch.Tensor, fmt: str, T):
    """(ft, odd) of each block of x (float64), as nested lists."""
    e, m, bias = FORMATS[fmt]
    emax = (1 << e) - 2 - bias
    M, C = x.shape
    a = torch.where(torch.isfinite(x), x.abs().clamp(max=limit(fmt, T)), 0.0)
    bad = ~torch.isfinite(x)
    ft, odd = [], []
    for r in range(0, M, ROWS):
        fr, orow = [], []
        for c in range(0, C, COLS):
            top = float(a[r:r + ROWS, c:c + COLS].max())
            fr.append(min(emax - _ceil_log2(top), MAX_FT) if top > 0 else 0)
            orow.append(bool(bad[r:r + ROWS, c:c + COLS].any()))
        ft.append(fr)
        odd.append(orow)
    return ft, odd


def spread(blocks, M: int, C: int, device="cpu") -> torch.Tensor:
    """Per-block values as a float64 [M][C]."""
    b = torch.as_tensor(blocks, dtype=torch.float64, device=device).view(-(-M // ROWS), -(-C // COLS))
    return b.repeat_interleave(ROWS, 0)[:M].repeat_interleave(COLS, 1)[:, :C]


def save(x: torch.Tensor, fmt: str, T):
    """Codes (uint8) and block words (int32) of x, a float64 CPU matrix."""
    e, m, _ = FORMATS[fmt]
    M, C = x.shape
    ft, odd = block_exponents(x, fmt, T)
    y = x.abs().clamp(max=limit(fmt, T)) * torch.exp2(spread(ft, M, C))
    vals = table(fmt)[:((1 << e) - 1) << m]  # the finite magnitudes, ascending
    hi = torch.searchsorted(vals, y.nan_to_num(0.0).contiguous()).clamp(max=len(vals) - 1)
    lo = (hi - 1).clamp(min=0)
    dl, dh = y - vals[lo], vals[hi] - y
    code = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    top = len(vals)
    code = torch.where(torch.isinf(x), top, torch.where(torch.isnan(x), top | (1 << (m - 1)), code))
    sign = torch.where(torch.isnan(x), 0, torch.signbit(x).long() * 128)
    words = [[(f & 0xFFFF) | (int(o) << 16) for f, o in zip(fr, orow)] for fr, orow in zip(ft, odd)]
    words = torch.tensor(words, dtype=torch.int32).view(-(-M // ROWS), -(-C // COLS))
    return (code | sign).to(torch.uint8), words


def load(codes: torch.Tensor, words: torch.Tensor, fmt: str) -> torch.Tensor:
    """The values of a checkpoint, float64."""
    M, C = codes.shape
    ft = words.to(torch.int64) & 0xFFFF
    ft = torch.where(ft >= 32768, ft - 65536, ft).double()
    return table(fmt).to(codes.device)[codes.long()] * torch.exp2(-spread(ft, M, C, codes.device))


def act(z: torch.Tensor, name: str) -> torch.Tensor:
    if name == "relu":
        return torch.where(z < 0, 0.0, z)
    if name == "gelu":
        return torch.where(z == -math.inf, 0.0, z * 0.5 * torch.special.erfc(-z / math.sqrt(2)))
    if name == "silu":
        return torch.where(z == -math.inf, 0.0, z / (1 + torch.exp(-z)))
    return z


def slope(z: torch.Tensor, name: str) -> torch.Tensor:
    if name == "none":
        return torch.ones_like(z)
    c = z.clamp(-700, 700)
    if name == "relu":
        d = (c > 0).double()
    elif name == "gelu":
        d = 0.5 * torch.special.erfc(-c / math.sqrt(2)) + c * torch.exp(-c * c / 2) / math.sqrt(2 * math.pi)
    else:
        s = 1 / (1 + torch.exp(-c))
        d = s + c * s / (1 + torch.exp(c))
    return torch.where(torch.isnan(z), math.nan, d)


# The largest |slope| of an activation, and a bound of its error in fp32 per
# unit of |z| (a handful of roundings and the special functions' own few ulps).
LIPSCHITZ = 1.13
ACT_ULPS = 16 * 2.0 ** -24


def sums_bound(absP: torch.Tensor, absQ: torch.Tensor, extra=0.0) -> torch.Tensor:
    """A bound of the error of fp32 sums over the last axis of Q and the first
    of P: each of the n additions is off by at most 2^-23 of the sum of
    magnitudes (a rounding towards zero would be), the products by half that
    (fp32 operands only)."""
    n = absQ.shape[1]
    return (n + 2) * 2.0 ** -23 * (absQ @ absP + extra)


def half_step(T) -> float:
    return torch.finfo(T).eps / 2


def tiny(T) -> float:
    """Half the smallest subnormal's step: the rounding error near zero."""
    return torch.finfo(T).smallest_normal * torch.finfo(T).eps / 2
