"""Operators of a mixture-of-experts layer on ciphertexts, as cases that can be
timed: layers over 8-bit floating-point weights, the same for requests that
name an expert and a bundle of inputs, and the gated sum of the experts' outputs.

Kinds:
  fp8      ckks_linear_mac_fp8: ciphertexts times e4m3 weights with one scale
           for every block of 128 inputs and `block_rows` outputs
  experts  ckks_experts_mac_fp8: requests, each one expert's layer over one
           bundle of ciphertexts, ragged in their number for each expert
  combine  ckks_experts_combine: sums of requests' outputs, each times the
           plaintext of its gates (one value a slot)

Where `own` is false the same results come from elementary torch operations.
All outputs are residues: whole numbers with one right value.  Residues are
below 2^30 and their products below 2^60, so the plain forms hold them in
64-bit integers, and in fp64 where every sum is exact.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False

WEIGHT_STD = 0.02       # trained projection weights are about this wide
BLOCK = 128             # inputs that share a scale
LARGEST = 448.0         # of e4m3


def listed():
    return [
        # The smallest layer, 16 features in a ring of 2^10: launch and latency.
        dict(name="fp8-16x16-n10", kind="fp8", log_n=10, limbs=2, log_scale=30, d_in=16, d_out=16, block_rows=128),
        # A router's scores: one output an expert.
        dict(name="fp8-1024x16-n13", kind="fp8", log_n=13, limbs=3, log_scale=31, d_in=1024, d_out=16, block_rows=128),
        # Odd sizes: one tensor-parallel share of a layer with a scale for each output.
        dict(name="fp8-513x1021-n13-rows", kind="fp8", log_n=13, limbs=3, log_scale=32, d_in=513, d_out=1021, block_rows=1),
        # A down projection: deep contraction, few outputs.
        dict(name="fp8-2048x768-n14", kind="fp8", log_n=14, limbs=4, log_scale=31, d_in=2048, d_out=768, block_rows=128),
        # An up projection in a large ring: the largest layer.
        dict(name="fp8-1024x2048-n15", kind="fp8", log_n=15, limbs=4, log_scale=31, d_in=1024, d_out=2048, block_rows=128),
        # A few small experts: the latency of a call.
        dict(name="experts-4-32x32-n10", kind="experts", log_n=10, limbs=2, log_scale=30, experts=4, count=5, padded=0,
             bundles=3, d_in=32, d_out=32, block_rows=128),
        # Odd sizes, a scale for each output, and room that the step does not fill.
        dict(name="experts-8-200x333-n11-rows", kind="experts", log_n=11, limbs=2, log_scale=32, experts=8, count=13,
             padded=3, bundles=6, d_in=200, d_out=333, block_rows=1),
        # Two experts for each of ten bundles, of sixteen fine-grained experts.
        dict(name="experts-16-1024x384-n12", kind="experts", log_n=12, limbs=3, log_scale=31, experts=16, count=20,
             padded=0, bundles=10, d_in=1024, d_out=384, block_rows=128),
        # Two experts' outputs for each of two bundles in a small ring: latency.
        dict(name="combine-2x16-n10", kind="combine", log_n=10, limbs=2, count=4, bundles=2, top=2, features=16),
        # Three experts a bundle, some bundles with fewer.
        dict(name="combine-5x37-n11", kind="combine", log_n=11, limbs=3, count=12, bundles=5, top=3, features=37),
        # The outputs of a layer of 256 features, two experts for each of six bundles.
        dict(name="combine-6x256-n13", kind="combine", log_n=13, limbs=3, count=12, bundles=6, top=2, features=256),
    ]


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _draw_once(rng):
    kind = rng.choice(["fp8", "fp8", "fp8", "experts", "experts", "experts", "combine", "combine"])
    c = dict(kind=kind, log_n=rng.randint(10, 16), limbs=rng.randint(1, 8))
    if kind == "combine":
        c.update(bundles=_spread(rng, 1, 64), top=rng.randint(1, 8), features=_spread(rng, 1, 2048))
        c["count"] = max(1, round(c["bundles"] * c["top"] * rng.uniform(0.4, 1.2)))
        return c
    c.update(log_scale=rng.randint(26, 36), d_in=_spread(rng, 1, 4096), d_out=_spread(rng, 1, 4096),
             block_rows=rng.choice([1, 64, 128, 128, 128]))
    if kind == "experts":
        c.update(experts=_spread(rng, 1, 64), count=_spread(rng, 1, 64), padded=rng.choice([0, 0, 1, 3]),
                 bundles=_spread(rng, 1, 32))
    return c


def draw(rng):
    while True:
        c = _draw_once(rng)
        w = work(c)
        # no larger than the largest listed case in traffic and in operations
        if w["bytes"] <= 3.2e9 and w["flops"] <= 1.1e12 and _state_bytes(c) <= 4e9:
            return c


def _requests(c):
    """(expert, bundle) of every request, the same for every seed: experts ascending, few of them with most of the
    requests and some with none; what is padded names no expert."""
    u = [((i + 1) * 2654435761 % (1 << 32)) / 2.0 ** 32 for i in range(c["count"])]
    expert = sorted(int(c["experts"] * v * v) for v in u) + [-1] * c["padded"]
    bundle = [i * 7 % c["bundles"] for i in range(c["count"])] + [0] * c["padded"]
    return expert, bundle


def _terms(c):
    """Requests whose outputs a bundle sums, the same for every seed: each request once while there are any, then none."""
    slots = c["bundles"] * c["top"]
    order = sorted(range(slots), key=lambda i: (i + 1) * 2654435761 % (1 << 32))
    flat = [-1] * slots
    for r, at in enumerate(order[: c["count"]]):
        flat[at] = r
    return np.array(flat, dtype=np.int32).reshape(c["bundles"], c["top"])


def _ct_words(c):
    return 2 * c["limbs"] << c["log_n"]


def _blocks(d_out, d_in, block_rows):
    return -(-d_out // block_rows), -(-d_in // BLOCK)


def _state_bytes(c):
    """Ciphertexts of the state, as the plain forms gather them."""
    if c["kind"] == "combine":
        return 4 * _ct_words(c) * c["features"] * (c["count"] + c["bundles"] * (1 + c["top"]))
    if c["kind"] == "fp8":
        return 4 * _ct_words(c) * (c["d_in"] + c["d_out"])
    rows = c["count"] + c["padded"]
    weights = 8 * (rows + c["experts"]) * c["limbs"] * c["d_in"] * c["d_out"]
    return 4 * _ct_words(c) * rows * (c["d_in"] + c["d_out"]) + weights


def work(case):
    words = _ct_words(case)
    if case["kind"] == "combine":
        used = int((_terms(case) >= 0).sum())
        # flops: one modular multiply-add is counted as two
        return {"bytes": 4 * words * case["features"] * (used + case["bundles"]) + 4 * words // 2 * used +
                4 * case["bundles"] * case["top"],
                "flops": 2 * used * case["features"] * words}
    d_in, d_out = case["d_in"], case["d_out"]
    rows, cols = _blocks(d_out, d_in, case["block_rows"])
    weights = d_in * d_out + 4 * rows * cols
    if case["kind"] == "fp8":
        return {"bytes": 4 * words * (d_in + d_out) + weights, "flops": 2 * d_out * d_in * words}
    expert, bundle = _requests(case)
    n = case["count"]
    return {"bytes": 4 * words * (len(set(bundle[:n])) * d_in + n * d_out) + len(set(expert[:n])) * weights + 8 * len(expert),
            "flops": 2 * n * d_out * d_in * words}


# ---- the modulus chain ------------------------------------------------------

def _is_prime(q):
    d, s = q - 1, 0
    while d % 2 == 0:
        d, s = d // 2, s + 1
    for a in (2, 3, 5, 7):  # deterministic below 3.2e9
        x = pow(a, d, q)
        if x in (1, q - 1):
            continue
        for _ in range(s - 1):
            x = x * x % q
            if x == q - 1:
                break
        else:
            return False
    return True


@functools.lru_cache(maxsize=None)
def _moduli(log_n, limbs):
    """The largest primes below 2^30 that are 1 mod 2N."""
    step = 2 << log_n
    q = ((1 << 30) - 1) // step * step + 1
    found = []
    while len(found) < limbs:
        if q < 1 << 30 and _is_prime(q):
            found.append(q)
        q -= step
    return tuple(found)


# ---- inputs -----------------------------------------------------------------

def _residues(g, prefix, qs, n):
    """int32 residues prefix + (L, n), limb l uniform below qs[l]."""
    out = torch.empty(tuple(prefix) + (len(qs), n), dtype=torch.int32, device="cuda")
    for l, q in enumerate(qs):
        out[..., l, :] = torch.randint(0, q, tuple(prefix) + (n,), generator=g, device="cuda", dtype=torch.int32)
    return out


def _weights(g, many, d_out, d_in, block_rows):
    """e4m3 weights [many][d_out][d_in] and their scales: the largest weight of a block is the largest number."""
    rows, cols = _blocks(d_out, d_in, block_rows)
    w = torch.zeros((many, rows * block_rows, cols * BLOCK), device="cuda")
    w[:, :d_out, :d_in] = torch.randn((many, d_out, d_in), generator=g, device="cuda") * WEIGHT_STD
    w = w.view(many, rows, block_rows, cols, BLOCK)
    scales = w.abs().amax((2, 4)) / LARGEST
    codes = (w / scales[:, :, None, :, None]).clamp_(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
    codes = codes.view(many, rows * block_rows, cols * BLOCK)[:, :d_out, :d_in].contiguous()
    return codes, scales.contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, L = 1 << case["log_n"], case["limbs"]
    qs = _moduli(case["log_n"], L)
    st = {"case": case, "q": torch.tensor(qs, dtype=torch.int64, device="cuda").view(L, 1)}
    if own:
        import paper_2606_17421_amd as ck
        st["ck"] = ck
        st["ctx"] = ck.Context(case["log_n"], L)
    if case["kind"] == "combine":
        st["terms"] = torch.from_numpy(_terms(case)).cuda()
        st["gates"] = _residues(g, (case["count"],), qs, n)
        st["ct"] = _residues(g, (case["count"], case["features"], 2), qs, n)
        if own:
            st["out"] = st["ck"].empty_u32((case["bundles"], case["features"], 2, L, n))
        return st
    d_in, d_out = case["d_in"], case["d_out"]
    if case["kind"] == "fp8":
        many, inputs, outputs = 1, (d_in, 2), (d_out, 2, L, n)
    else:
        many, inputs, outputs = case["experts"], (case["bundles"], d_in, 2), (case["count"] + case["padded"], d_out, 2, L, n)
        expert, bundle = _requests(case)
        st["expert"] = torch.tensor(expert, dtype=torch.int32, device="cuda")
        st["bundle"] = torch.tensor(bundle, dtype=torch.int32, device="cuda")
        st["out"] = torch.zeros(outputs, dtype=torch.int32, device="cuda")  # what is padded stays as it is
    st["w8"], st["scales"] = _weights(g, many, d_out, d_in, case["block_rows"])
    st["ct"] = _residues(g, inputs, qs, n)
    if own:
        ck, ctx = st["ck"], st["ctx"]
        need = ck.ckks_fp8_weight_bytes(ctx, d_out, d_in, L)
        st["enc"] = ck.empty_workspace(many * need).view(many, -1)
        for e in range(many):
            ck.ckks_linear_encode_fp8(ctx, st["w8"][e], st["scales"][e], d_out, d_in, case["block_rows"], L,
                                      float(1 << case["log_scale"]), st["enc"][e])
        if case["kind"] == "fp8":
            st["out"] = ck.empty_u32(outputs)
    return st


# ---- one pass ---------------------------------------------------------------

def run(state):
    return _RUN[state["case"]["kind"]](state)


def _plaintexts(st):
    """64 times the weights, rounded to whole numbers, times the rounded scales: residues [many][L][d_out][d_in]."""
    c, q = st["case"], st["q"]
    v = torch.round(st["w8"].to(torch.float32) * 64).to(torch.int64)
    s = torch.round(st["scales"].double() * (2.0 ** c["log_scale"] / 64)).to(torch.int64)
    row = torch.arange(c["d_out"], device="cuda") // c["block_rows"]
    col = torch.arange(c["d_in"], device="cuda") // BLOCK
    s = s[:, row][:, :, col]
    m = q[None, :, :, None]
    return v[:, None].remainder(m).mul_(s[:, None].remainder(m)).remainder_(m)


def _products(w, x, q):
    """w [batch][d_out][d_in] times x [batch][d_in][columns] mod q [batch][1][1].  Halves of 15 bits: every product of
    two matrices is exact in fp64 (2^30 d_in < 2^53)."""
    wh, wl = (w >> 15).double(), (w & 32767).double()
    xh, xl = (x >> 15).double(), (x & 32767).double()
    out = torch.bmm(wh, xh).to(torch.int64).remainder_(q).mul_(1 << 15)
    out += torch.bmm(wh, xl).add_(torch.bmm(wl, xh)).to(torch.int64)
    out = out.remainder_(q).mul_(1 << 15)
    out += torch.bmm(wl, xl).to(torch.int64)
    return out.remainder_(q).to(torch.int32)


def _run_fp8(st):
    c = st["case"]
    d_in, d_out, L = c["d_in"], c["d_out"], c["limbs"]
    if own:
        st["ck"].ckks_linear_mac_fp8(st["ctx"], st["enc"][0], st["ct"], st["out"], d_out, d_in, L)
        return st["out"]
    x = st["ct"].permute(2, 0, 1, 3).reshape(L, d_in, -1)                            # [L][d_in][2 N]
    out = _products(_plaintexts(st)[0], x, st["q"][:, :, None])
    return out.view(L, d_out, 2, -1).permute(1, 2, 0, 3).contiguous()


def _run_experts(st):
    c = st["case"]
    d_in, d_out, L = c["d_in"], c["d_out"], c["limbs"]
    if own:
        st["ck"].ckks_experts_mac_fp8(st["ctx"], st["enc"], st["expert"], st["bundle"], st["ct"], st["out"], d_out, d_in, L)
        return st["out"]
    rows = len(st["expert"])
    w = _plaintexts(st)[st["expert"].clamp(min=0).to(torch.int64)]                   # [rows][L][d_out][d_in]
    x = st["ct"][st["bundle"].to(torch.int64)].permute(0, 3, 1, 2, 4)                # [rows][L][d_in][2][N]
    out = _products(w.view(rows * L, d_out, d_in), x.reshape(rows * L, d_in, -1), st["q"].repeat(rows, 1)[:, :, None])
    out = out.view(rows, L, d_out, 2, -1).permute(0, 2, 3, 1, 4)
    st["out"].copy_(torch.where((st["expert"] >= 0).view(-1, 1, 1, 1, 1), out, st["out"]))
    return st["out"]


def _run_combine(st):
    c = st["case"]
    if own:
        st["ck"].ckks_experts_combine(st["ctx"], st["gates"], st["ct"], st["terms"], st["out"], c["features"], c["limbs"])
        return st["out"]
    at = st["terms"].clamp(min=0).to(torch.int64)                                    # [bundles][top]
    gates = st["gates"].to(torch.int64)[at] * (st["terms"] >= 0)[:, :, None, None]   # [bundles][top][L][N]
    out = st["ct"][at].to(torch.int64).mul_(gates[:, :, None, None]).remainder_(st["q"])
    return out.sum(1).remainder_(st["q"]).to(torch.int32)


_RUN = {"fp8": _run_fp8, "experts": _run_experts, "combine": _run_combine}


# ---- the definitions --------------------------------------------------------

def exact(case, seed):
    """From the definitions in 64-bit integers, entry by entry; None for cases that take too long."""
    w = work(case)
    if own or w["bytes"] > 6e7 or w["flops"] > 2e9:
        return None
    if case["kind"] != "combine" and case["d_in"] * case["d_out"] * case.get("count", 1) > 2e5:  # a step for each weight
        return None
    st = prepare(case, seed)
    q = np.array(_moduli(case["log_n"], case["limbs"]), dtype=np.int64)
    if case["kind"] == "combine":
        return _exact_combine(case, st, q)
    codes = st["w8"].view(torch.uint8).cpu().numpy()
    scales, x = st["scales"].cpu().numpy(), st["ct"].cpu().numpy().astype(np.int64)
    if case["kind"] == "fp8":
        return torch.from_numpy(_exact_layer(case, codes[0], scales[0], x, q))
    out = st["out"].cpu().numpy()
    for r, (e, b) in enumerate(zip(*_requests(case))):
        if e >= 0:
            out[r] = _exact_layer(case, codes[e], scales[e], x[b], q)
    return torch.from_numpy(out)


def _e4m3(code):
    """64 times the number that a code stands for (a sign, four bits of exponent, three of mantissa, the least step
    2^-9), rounded half to even."""
    sign, exponent, mantissa = code >> 7, code >> 3 & 15, code & 7
    eighths = mantissa if exponent == 0 else (8 + mantissa) << (exponent - 1)
    size, rest = divmod(eighths, 8)
    size += rest > 4 or (rest == 4 and size % 2 == 1)
    return -size if sign else size


def _exact_layer(case, codes, scales, x, q):
    out = np.zeros((case["d_out"],) + x.shape[1:], dtype=np.int64)
    for j in range(case["d_out"]):
        for i in range(case["d_in"]):
            s = float(scales[j // case["block_rows"], i // BLOCK]) * 2.0 ** case["log_scale"] / 64
            weight = _e4m3(int(codes[j, i])) * int(np.rint(s))
            weight = np.array([weight % int(v) for v in q], dtype=np.int64)
            out[j] = (out[j] + weight[None, :, None] * x[i]) % q[None, :, None]
    return out.astype(np.int32)


def _exact_combine(case, st, q):
    gates, y = st["gates"].cpu().numpy().astype(np.int64), st["ct"].cpu().numpy().astype(np.int64)
    out = np.zeros((case["bundles"],) + y.shape[1:], dtype=np.int64)
    for t, terms in enumerate(_terms(case)):
        for r in terms:
            if r >= 0:
                out[t] = (out[t] + gates[r][None, None] * y[r]) % q[:, None]
    return torch.from_numpy(out.astype(np.int32))
