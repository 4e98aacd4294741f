"""A mixture-of-experts layer on encrypted tokens, on one GPU.

    python examples/encrypted_experts.py

Two bundles of tokens (one ciphertext a feature, a slot a token) are encrypted.
The trusted side has routed every token to two of the experts; a bundle goes to
each expert that any of its tokens has, as one request, and the requests of all
experts are one call over e4m3 weights with a scale a block.  The outputs are
rescaled and summed for each bundle, every expert's times the encoded gates of
its slots (zero for tokens that are not its own), rescaled again, decrypted
and compared with the layer in floating point: over the weights that are encoded, within the
noise, and over the quantised weights, scales times e4m3 numbers, within that and the encoding's rounding.
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_17421_amd as ck  # noqa: E402

LOG_N, LIMBS = 10, 4
SCALE_X, SCALE_W, SCALE_G = float(1 << 25), float(1 << 31), float(1 << 28)
D_IN, D_OUT, EXPERTS, BUNDLES, TOP, ROOM = 200, 40, 4, 2, 2, 10
BLOCK_ROWS, BLOCK, LARGEST = 32, 128, 448.0


def quantise(w):
    """Block-maximum quantisation to e4m3: (weights, scales, the weights that the encoded layer stands for, the quantised
    weights, how far the two may be apart)."""
    d_out, d_in = w.shape
    row, col = np.arange(d_out) // BLOCK_ROWS, np.arange(d_in) // BLOCK
    scales = np.zeros((row[-1] + 1, col[-1] + 1), np.float32)
    np.maximum.at(scales, (row[:, None], col[None, :]), (np.abs(w) / LARGEST).astype(np.float32))
    w8 = torch.from_numpy(w / scales[row][:, col]).clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
    f, s = w8.to(torch.float64).numpy(), scales.astype(np.float64)[row][:, col]
    units = np.rint(64 * f) * np.rint(s * (SCALE_W / 64))
    # a number is a multiple of 1/64 from 1/8 on, and a scale is rounded to a multiple of 64 / SCALE_W
    apart = np.where(np.abs(f) < 0.125, s / 128, 0) + np.abs(np.rint(64 * f)) / (2 * SCALE_W)
    return w8, scales, units / SCALE_W, s * f, apart


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

    # the secret, and the experts' weights encoded once
    s = rng.integers(-1, 2, n)
    s_ntt = ck.to_device(np.stack([np.mod(s, p) for p in q]).astype(np.uint32))
    ck.ckks_ntt(ctx, s_ntt, 1, LIMBS)
    bad, weights, quantised, apart = ints([0]), [], [], []
    w_fp8 = ck.empty_workspace(EXPERTS * ck.ckks_fp8_weight_bytes(ctx, D_OUT, D_IN, LIMBS)).view(EXPERTS, -1)
    for e in range(EXPERTS):
        w8, scales, w, sf, far = quantise(rng.normal(0, 0.02, (D_OUT, D_IN)))
        ck.ckks_linear_encode_fp8(ctx, w8.cuda(), ck.to_device(scales), D_OUT, D_IN, BLOCK_ROWS, LIMBS, SCALE_W, w_fp8[e], bad)
        assert int(bad) == 0
        weights.append(w)
        quantised.append(sf)
        apart.append(far)

    # two bundles of tokens; their gates: two experts a token, of the second bundle's tokens none the last
    x = rng.uniform(-1, 1, (BUNDLES, D_IN, n // 2))
    scores = rng.normal(0, 1, (BUNDLES, EXPERTS, n // 2))
    scores[1, EXPERTS - 1] = -np.inf
    kept = np.sort(scores, axis=1)[:, -TOP][:, None]
    gates = np.where(scores >= kept, np.exp(scores), 0)
    gates /= gates.sum(axis=1, keepdims=True)

    pt, ct = ck.empty_u32((BUNDLES * D_IN, LIMBS, n)), ck.empty_u32((BUNDLES, D_IN, 2, LIMBS, n))
    ck.ckks_linear_encode_poly(ctx, ck.to_device(x.reshape(-1, n // 2)), BUNDLES * D_IN, LIMBS, SCALE_X, pt)
    a = np.stack([rng.integers(0, p, (BUNDLES * D_IN, n)) for p in q], axis=1).astype(np.uint32)
    e = np.rint(rng.normal(0, 3.2, (BUNDLES * D_IN, n))).clip(-19, 19).astype(np.int32)
    ck.ckks_encrypt(ctx, pt, s_ntt, ck.to_device(a), ck.to_device(e), BUNDLES * D_IN, LIMBS, ct)

    # requests in expert order; the call has room for more than there are
    requests = [(k, b) for k in range(EXPERTS) for b in range(BUNDLES) if gates[b, k].any()]
    padded = requests + [(-1, 0)] * (ROOM - len(requests))
    out, status = ck.empty_u32((ROOM, D_OUT, 2, LIMBS, n)), ints([-1] * ROOM)
    out.zero_()
    ck.ckks_experts_mac_fp8(ctx, w_fp8, ints([r[0] for r in padded]), ints([r[1] for r in padded]), ct, out, D_OUT, D_IN, LIMBS,
                            status)
    y = ck.empty_u32((ROOM, D_OUT, 2, LIMBS - 1, n))
    ck.ckks_rescale(ctx, out, y, ROOM * D_OUT, LIMBS)
    scale_y = ck.ckks_rescaled_scale(ctx, SCALE_X * SCALE_W, LIMBS)

    # the gated sums
    g = np.zeros((ROOM, n // 2))
    terms = np.full((BUNDLES, EXPERTS), -1)
    for r, (k, b) in enumerate(requests):
        g[r] = gates[b, k]
        terms[b, k] = r
    g_pt = ck.empty_u32((ROOM, LIMBS - 1, n))
    ck.ckks_linear_encode_poly(ctx, ck.to_device(g), ROOM, LIMBS - 1, SCALE_G, g_pt)
    total, z = ck.empty_u32((BUNDLES, D_OUT, 2, LIMBS - 1, n)), ck.empty_u32((BUNDLES, D_OUT, 2, LIMBS - 2, n))
    ck.ckks_experts_combine(ctx, g_pt, y, ints(terms.tolist()), total, D_OUT, LIMBS - 1)
    ck.ckks_rescale(ctx, total, z, BUNDLES * D_OUT, LIMBS - 1)
    scale_z = ck.ckks_rescaled_scale(ctx, scale_y * SCALE_G, LIMBS - 1)

    # the trusted side's read
    m = ck.empty_u32((BUNDLES * D_OUT, LIMBS - 2, n))
    ck.ckks_decrypt(ctx, z, s_ntt, BUNDLES * D_OUT, LIMBS - 2, m)
    got = slots_of(ck.to_host_u32(m), q, scale_z, n).real.reshape(BUNDLES, D_OUT, n // 2)
    each = np.stack([[weights[k] @ x[b] for k in range(EXPERTS)] for b in range(BUNDLES)])      # [bundle][expert][D_OUT][N/2]
    want = (each * gates[:, :, None]).sum(axis=1)
    # A polynomial with independent coefficients of variance v has variance N v / 2 in the real part of a slot.  A
    # rescale rounds both components: tau0 + tau1 s with tau uniform in +-1/2; encryption adds errors of 3.2, and each
    # encoding rounds by at most 1/2.
    power = np.array([pow(5, j, 2 * n) for j in range(n // 2)])
    s_at = np.exp(1j * np.pi * (power[:, None] * np.arange(n) % (2 * n)) / n) @ s
    rescale = n / 24 * (1 + np.abs(s_at) ** 2)
    wide = np.stack([(w ** 2).sum(axis=1) for w in weights])                                     # [expert][D_OUT]
    var_each = rescale / scale_y ** 2 + (wide * n / 2 * (3.2 ** 2 + 1 / 12) / SCALE_X ** 2)[..., None]
    var = ((gates ** 2)[:, :, None] * var_each[None]).sum(axis=1) + rescale / scale_z ** 2
    var = var + (each ** 2).sum(axis=1) * n / 24 / SCALE_G ** 2
    off = np.abs(got - want)
    # against the quantised weights: six standard deviations and the encoding's rounding, |x| <= 1
    layer = np.stack([(np.stack([sf @ x[b] for sf in quantised]) * gates[b][:, None]).sum(axis=0) for b in range(BUNDLES)])
    rounding = np.stack([(np.stack([far.sum(axis=1) for far in apart])[:, :, None] * gates[b][:, None]).sum(axis=0) for b in range(BUNDLES)])
    from_layer = np.abs(got - layer) / (6 * np.sqrt(var) + rounding)
    result = {"requests": len(requests), "status": status.tolist(), "largest": float(np.abs(want).max()),
              "worst_error": float(off.max()), "worst_over_sd": float((off / np.sqrt(var)).max()),
              "worst_from_layer": float(from_layer.max()), "largest_rounding": float(rounding.max())}
    ctx.close()
    return result


if __name__ == "__main__":
    print(main())
