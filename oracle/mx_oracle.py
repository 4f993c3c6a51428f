"""CPU oracle of the microscaled 4-bit format (numpy, 64 bits): quantisation, packing, expansion and products from their definition.
Only tests/ and ``__graft_entry__.smoke()`` may import it."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK, ROW = 32, 128


def to_double(bits: np.ndarray, kind: str) -> np.ndarray:
    """numbers of the bit patterns of "f16" / "bf16" (uint16) or "f32" (uint32)"""
    if kind == "f16":
        return bits.view(np.float16).astype(np.float64)
    if kind == "bf16":
        return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    return bits.view(np.float32).astype(np.float64)


def from_double(v: np.ndarray, kind: str) -> np.ndarray:
    """bit patterns of the nearest numbers of the type (ties to even; NaN stays NaN)"""
    with np.errstate(over="ignore"):
        if kind == "f16":
            return v.astype(np.float16).view(np.uint16)
        if kind == "f32":
            return v.astype(np.float32).view(np.uint32)
        # bf16: exact for the values used here unless fp32 already rounds (numbers below 2^-126)
        u = v.astype(np.float32).view(np.uint32)
        r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
        return np.where(np.isnan(v), np.uint16(0x7FC0), r)


def padded(n: int) -> int:
    return -(-n // ROW) * ROW


def quantize(v: np.ndarray):
    """(codes [M, P] 0..15, scale bytes [M, P / 32]) of the rows of v (64 bits)"""
    M, N = v.shape
    w = np.zeros((M, padded(N)))
    w[:, :N] = v
    w = w.reshape(M, -1, BLOCK)
    bad = ~np.isfinite(w).all(axis=2)
    w = np.where(bad[:, :, None], 0.0, w)
    top = np.abs(w).max(axis=2)
    e = np.where(top > 0, np.frexp(top)[1] - 1 - 2, -127)
    e = np.clip(e, -127, None)
    t = np.abs(w) * np.ldexp(1.0, -e)[:, :, None]
    d = np.abs(t[..., None] - GRID)                                   # nearest grid value; of two, the one with the even code
    lo = d.argmin(axis=3)
    other = np.minimum(lo + 1, 7)
    tie = (other != lo) & (np.take_along_axis(d, other[..., None], 3)[..., 0] == np.take_along_axis(d, lo[..., None], 3)[..., 0])
    code = np.where(tie & (lo % 2 == 1), other, lo)
    code = code | np.where(np.signbit(w), 8, 0)
    code = np.where(bad[:, :, None], 0, code)
    return code.reshape(M, -1).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def pack(code: np.ndarray) -> np.ndarray:
    return code[:, 0::2] | (code[:, 1::2] << 4)


def expand(packed: np.ndarray, scales: np.ndarray, N: int) -> np.ndarray:
    code = np.stack([packed & 15, packed >> 4], axis=2).reshape(packed.shape[0], -1)
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    f = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return (v.reshape(v.shape[0], -1, BLOCK) * f[:, :, None]).reshape(v.shape[0], -1)[:, :N]
