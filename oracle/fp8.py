"""Layers over 8-bit floating-point weights and gated sums of their outputs (CPU
oracle; test infrastructure only).

A weight is scales[j // block_rows, i // 128] f[j, i] with f an e4m3 number.  Its
plaintext is the integer rint(64 f) rint(scales * scale / 64), both rounded half to
even, so the layer is the scalar-weight MAC (section 3.2) over those integers mod
each prime.  Python integers throughout: scaled scales may be as large as 2^63.

Parity: pinned (tests/test_oracle_fp8.py) by the numbers of e4m3 written out, by a
tiny case, and by the scalar encode where both round alike.
"""
from __future__ import annotations

import numpy as np

from .linear import mac_scalar

BLOCK = 128


def numbers(codes) -> np.ndarray:
    """e4m3 codes -> float64: (-1)^s 2^(e - 7) (1 + m / 8), or (-1)^s 2^-6 m / 8 where e = 0; NaN for e = 15, m = 7."""
    c = np.asarray(codes, np.uint8).astype(np.int64)
    e, m = c >> 3 & 15, c & 7
    f = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7.0))
    f = np.where((e == 15) & (m == 7), np.nan, f)
    return np.where(c >> 7, -f, f)


def plaintexts(codes, scales, block_rows: int, scale: float) -> np.ndarray:
    """The integers rint(64 f) rint(scales * scale / 64), as Python integers (object array d_out x d_in); NaN weights
    and scales that are NaN, infinite or scaled to 2^63 and more are zero."""
    f = numbers(codes)
    v = np.rint(64 * np.nan_to_num(f, nan=0.0)).astype(np.int64)
    s = np.asarray(scales, np.float32).astype(np.float64)
    s = np.where(np.isfinite(s), s, 0.0) * (scale / 64)
    s = np.rint(np.where(abs(s) < 2.0 ** 63, s, 0.0))
    s = np.vectorize(int, otypes=[object])(s) if s.size else s.astype(object)
    row, col = np.arange(v.shape[0]) // block_rows, np.arange(v.shape[1]) // BLOCK
    return v.astype(object) * s[row][:, col]


def units(codes) -> np.ndarray:
    """The largest u of 64, 128, 256 and 512 with |u f| <= 28672 for all weights of a row and block (d_out, blocks)."""
    f = np.abs(np.nan_to_num(numbers(codes), nan=0.0))
    top = np.stack([f[:, b:b + BLOCK].max(axis=1) for b in range(0, f.shape[1], BLOCK)], axis=1)
    return np.select([u * top <= 28672 for u in (512, 256, 128)], [512, 256, 128], 64)


def plaintexts_in_units(codes, scales, block_rows: int, scale: float) -> np.ndarray:
    """The integers rint(u f) rint(scales * scale / u); zero as in plaintexts, and where a scale rounds to zero for u = 512."""
    f = np.nan_to_num(numbers(codes), nan=0.0)
    row, col = np.arange(f.shape[0]) // block_rows, np.arange(f.shape[1]) // BLOCK
    s = np.asarray(scales, np.float32).astype(np.float64)
    s = np.where(np.isfinite(s), s, 0.0) * scale
    s = np.where((abs(s / 64) < 2.0 ** 63) & (np.rint(s / 512) != 0), s, 0.0)[row][:, col]
    u = units(codes)[:, col]
    v, whole = np.rint(u * f).astype(np.int64), np.rint(s / u)
    return v.astype(object) * np.vectorize(int, otypes=[object])(whole)


def rounded(codes) -> int:
    """How many weights plaintexts_in_units does not keep."""
    f = np.nan_to_num(numbers(codes), nan=0.0)
    x = units(codes)[:, np.arange(f.shape[1]) // BLOCK] * f
    return int((x != np.rint(x)).sum())


def residues(p, qs) -> np.ndarray:
    """Integers (d_out, d_in) -> uint64 (d_out, d_in, L)."""
    return np.stack([(p % int(q)).astype(np.uint64) for q in qs], axis=-1)


def mac(codes, scales, ct, block_rows: int, scale: float, qs, rows=None, in_units: bool = False) -> np.ndarray:
    """ct (d_in, 2, L, N) residues -> (len(rows), 2, L, N)."""
    integers = plaintexts_in_units if in_units else plaintexts
    return mac_scalar(residues(integers(codes, scales, block_rows, scale), qs), ct, qs, rows=rows)


def combine(gates, y, terms, qs) -> np.ndarray:
    """gates (count, L, N), y (count, features, 2, L, N), terms (bundles, top) -> (bundles, features, 2, L, N)."""
    gates, y = np.asarray(gates).astype(np.uint64), np.asarray(y).astype(np.uint64)
    q = np.array(qs, np.uint64)[:, None]
    out = np.zeros((len(terms),) + y.shape[1:], np.uint64)
    for t, row in enumerate(terms):
        for r in row:
            if 0 <= r < len(y):
                out[t] = (out[t] + gates[r] * y[r] % q) % q
    return out
