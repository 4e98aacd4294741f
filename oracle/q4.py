"""Layers over 4-bit weights (CPU oracle; test infrastructure only).

A weight is scales[j, i // group] (u[j, i] - z[j, i // group]) with u in 0..15 and
z = 8 where there are no zero points.  Its plaintext is the integer (u - z)
rint(scales * scale), rounded half to even, so the layer is the scalar-weight
MAC (section 3.2) over those integers mod each prime.  Python integers
throughout: scaled scales may be as large as 2^63.

Parity: pinned (tests/test_oracle_q4.py) by a written-out tiny case, by the
nibble order, and by the scalar encode where the scales are exact.
"""
from __future__ import annotations

import numpy as np

from .linear import mac_scalar


def unpack(w4, d_in: int) -> np.ndarray:
    """uint8 (d_out, (d_in + 1) // 2), the even input in the low half -> int64 (d_out, d_in)."""
    w4 = np.asarray(w4, dtype=np.uint8)
    both = np.stack([w4 & 15, w4 >> 4], axis=-1).reshape(w4.shape[0], -1)
    return both[:, :d_in].astype(np.int64)


def pack(u) -> np.ndarray:
    """int (d_out, d_in) in 0..15 -> uint8 (d_out, (d_in + 1) // 2)."""
    u = np.asarray(u, dtype=np.uint8)
    if u.shape[1] % 2:
        u = np.concatenate([u, np.zeros((u.shape[0], 1), np.uint8)], axis=1)
    return (u[:, 0::2] | (u[:, 1::2] << 4)).astype(np.uint8)


def plaintexts(w4, scales, zeros, d_in: int, group: int, scale: float) -> np.ndarray:
    """The integers (u - z) rint(scales * scale), as Python integers (object array d_out x d_in)."""
    u = unpack(w4, d_in)
    of = np.arange(d_in) // group
    z = np.full(np.shape(scales), 8, np.int64) if zeros is None else np.asarray(zeros, np.int64) & 15
    s = np.rint(np.asarray(scales, np.float32).astype(np.float64) * scale)
    s = np.vectorize(int, otypes=[object])(s) if s.size else s.astype(object)
    return (u - z[:, of]).astype(object) * s[:, of]


def residues(p, qs) -> np.ndarray:
    """Integers (d_out, d_in) -> uint64 (d_out, d_in, L)."""
    return np.stack([(p % int(q)).astype(np.uint64) for q in qs], axis=-1)


def mac(w4, scales, zeros, ct, group: int, scale: float, qs, rows=None) -> np.ndarray:
    """ct (d_in, 2, L, N) residues -> (len(rows), 2, L, N)."""
    p = plaintexts(w4, scales, zeros, np.asarray(ct).shape[0], group, scale)
    return mac_scalar(residues(p, qs), ct, qs, rows=rows)
