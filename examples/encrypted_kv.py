"""Encrypted keys and values of a decoding server, on one GPU.

    python examples/encrypted_kv.py

A prompt's hidden states are encrypted one ciphertext a feature (a slot a
request lane); the K and V projections, stacked as one layer of 4-bit weights,
turn each token's ciphertexts into its row of the cache; the rows are appended
to a paged sequence, the sequence is forked into two continuations that share its
pages, each continuation gets a token of its own, the prompt ends and the pool is
compacted, and the trusted side decrypts the continuations through the page
table and compares them with the projections in floating point.
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_17421_amd as ck  # noqa: E402

LOG_N, LIMBS, SCALE = 10, 3, float(1 << 25)
D, D_KV, GROUP, PROMPT = 64, 16, 32, 6
PAGES, PAGE_ROWS, SEQS, MAX_PAGES = 12, 4, 3, 4


def quantise(w, group):
    """Absolute-maximum quantisation: (packed 4-bit u, scales, the weights that they stand for)."""
    d_out, d_in = w.shape
    g = w.reshape(d_out, d_in // group, group)
    scales = (np.abs(g).max(axis=2) / 7).astype(np.float32)
    u = (np.rint(g / scales[:, :, None]).clip(-8, 7) + 8).astype(np.uint8)
    stands_for = ((u.astype(np.float64) - 8) * scales[:, :, None]).reshape(d_out, d_in)
    u = u.reshape(d_out, d_in)
    return u[:, 0::2] | (u[:, 1::2] << 4), scales, stands_for


def slots_of(residues, q, scale, n):
    """Coefficient residues [..][2][N] below q0, q1 -> slot values [..][N/2]."""
    r0, r1 = (residues[..., l, :].astype(np.int64) for l in range(2))
    k = (r1 - r0) % q[1] * pow(q[0], -1, q[1]) % q[1]
    x = r0 + q[0] * k                                         # below q0 q1 < 2^60
    m = np.where(x > q[0] * q[1] // 2, x - q[0] * q[1], x) / scale
    power = np.array([pow(5, j, 2 * n) for j in range(n // 2)])
    return m @ np.exp(1j * np.pi * (power[:, None] * np.arange(n) % (2 * n)) / n).T


def main(seed: int = 0) -> dict:
    ctx = ck.Context(LOG_N, LIMBS)
    n, q = ctx.n, ctx.moduli
    rng = np.random.default_rng(seed)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731

    # the secret, and the K and V weights encoded once
    s = rng.integers(-1, 2, n)
    s_ntt = ck.to_device(np.stack([np.mod(s, p) for p in q]).astype(np.uint32))
    ck.ckks_ntt(ctx, s_ntt, 1, LIMBS)
    w4, scales, w = quantise(rng.normal(0, 0.02, (2 * D_KV, D)), GROUP)
    w_q4 = ck.empty_workspace(ck.ckks_q4_weight_bytes(ctx, 2 * D_KV, D, GROUP, LIMBS))
    ck.ckks_linear_encode_q4(ctx, ck.to_device(w4), ck.to_device(scales), None, 2 * D_KV, D, GROUP, LIMBS, SCALE, w_q4)

    def project(x):
        """Hidden states [D][N/2] of one token -> its encrypted K and V row."""
        pt, ct = ck.empty_u32((D, LIMBS, n)), ck.empty_u32((D, 2, LIMBS, n))
        ck.ckks_linear_encode_poly(ctx, ck.to_device(x), D, LIMBS, SCALE, pt)
        a = np.stack([rng.integers(0, p, (D, n)) for p in q], axis=1).astype(np.uint32)
        e = np.rint(rng.normal(0, 3.2, (D, n))).clip(-19, 19).astype(np.int32)
        ck.ckks_encrypt(ctx, pt, s_ntt, ck.to_device(a), ck.to_device(e), D, LIMBS, ct)
        mac, row = ck.empty_u32((2 * D_KV, 2, LIMBS, n)), ck.empty_u32((2 * D_KV, 2, LIMBS - 1, n))
        ck.ckks_linear_mac_q4(ctx, w_q4, ct, mac, 2 * D_KV, D, GROUP, LIMBS)
        ck.ckks_rescale(ctx, mac, row, 2 * D_KV, LIMBS)
        return row

    cache = ck.Cache.empty(ctx, PAGES, PAGE_ROWS, 2 * D_KV, LIMBS - 1, SEQS, MAX_PAGES)
    status = ints([0, 0])

    def append(seq, row0, rows):
        ws = ck.empty_workspace(ck.ckks_cache_workspace_bytes(ctx, cache, ck.CKKS_CACHE_APPEND, len(seq), len(rows)))
        ck.ckks_cache_append(ctx, cache, seq, row0, rows, ws, status)

    # the prompt, its two continuations, and the prompt's end
    prompt = rng.uniform(-1, 1, (PROMPT, D, n // 2))
    append(ints([0]), ints([0, PROMPT]), torch.stack([project(x) for x in prompt]))
    ck.ckks_cache_fork(ctx, cache, ints([0, 0]), ints([1, 2]), status)
    nexts = rng.uniform(-1, 1, (2, D, n // 2))
    append(ints([1, 2]), None, torch.stack([project(x) for x in nexts]))
    held = int((cache.refs > 0).sum())
    ck.ckks_cache_free(ctx, cache, ints([0]))
    live = ints([0])
    ck.ckks_cache_compact(ctx, cache, live, ck.empty_workspace(ck.ckks_cache_workspace_bytes(ctx, cache, ck.CKKS_CACHE_COMPACT)))

    # the trusted side's read of both continuations
    rows = PROMPT + 1
    seq, pos = ints([1] * rows + [2] * rows), ints(list(range(rows)) * 2)
    m = ck.empty_u32((2 * rows, 2 * D_KV, LIMBS - 1, n))
    ck.ckks_cache_decrypt(ctx, cache, seq, pos, s_ntt, m)
    scale_out = ck.ckks_rescaled_scale(ctx, SCALE * SCALE, LIMBS)
    got = slots_of(ck.to_host_u32(m), q, scale_out, n)
    want = np.stack([w @ x for i in range(2) for x in [*prompt, nexts[i]]])
    # The rescale rounds both components: tau0 + tau1 s with coefficients uniform in +-1/2, whose value at
    # slot j has a standard deviation of sqrt(N/24 (1 + |s(zeta_j)|^2)) units of the output scale.
    power = np.array([pow(5, j, 2 * n) for j in range(n // 2)])
    s_at = np.exp(1j * np.pi * (power[:, None] * np.arange(n) % (2 * n)) / n) @ s
    sd = np.sqrt(n / 24 * (1 + np.abs(s_at) ** 2)) / scale_out
    out = {"rows": 2 * rows, "held_before": held, "held_after": int(live.item()), "status": status.tolist(),
           "worst_error": float(np.abs(got.real - want).max()), "worst_over_sd": float((np.abs(got.real - want) / sd).max())}
    ctx.close()
    return out


if __name__ == "__main__":
    print(main())
