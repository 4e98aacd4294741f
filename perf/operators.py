"""Operators around an encrypted K/V projection, as cases that can be timed:
the linear layer over 4-bit group-scaled weights and the paged cache of
ciphertext rows that its outputs are kept in.

Kinds:
  q4       ckks_linear_mac_q4: ciphertexts times 4-bit weights with one scale
           (and zero point) a group of inputs
  step     one decoding step of forked sequences: ckks_cache_fork of prompts
           into branches (the branches of the pass before are released),
           ckks_cache_append of new rows to every branch
  compact  ckks_cache_free of finished sequences, then ckks_cache_compact
  gather   ckks_cache_gather of the rows of sequences
  decrypt  ckks_cache_decrypt of the rows of sequences

Where `own` is false the same results come from elementary torch operations.
All outputs are residues, pages and counts: whole numbers with one right
value.  Residues are below 2^30 and their products below 2^60, so the plain
forms hold them in 64-bit integers, and in fp64 where every sum is exact.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False

WEIGHT_STD = 0.02       # trained projection weights are about this wide
KINDS = ("q4", "step", "compact", "gather", "decrypt")


def listed():
    return [
        # The smallest layer, 16 features in a ring of 2^10: launch and latency.
        dict(name="q4-16x16-n10", kind="q4", log_n=10, limbs=2, log_scale=25, d_in=16, d_out=16, group=32, zeros=False),
        # A down projection (deep contraction, few outputs), group 64 with zero points.
        dict(name="q4-3072x768-n14-zeros", kind="q4", log_n=14, limbs=4, log_scale=26, d_in=3072, d_out=768, group=64,
             zeros=True),
        # Odd sizes: one tensor-parallel share of a layer, the last group ragged.
        dict(name="q4-513x1021-n13-zeros", kind="q4", log_n=13, limbs=3, log_scale=26, d_in=513, d_out=1021, group=32,
             zeros=True),
        # GPT-2-124M FFN up projection: the largest layer.
        dict(name="q4-768x3072-n15", kind="q4", log_n=15, limbs=6, log_scale=26, d_in=768, d_out=3072, group=128,
             zeros=False),
        # One prompt forked in two in a small ring: the latency of a step.
        dict(name="step-2-branches-n10", kind="step", log_n=10, limbs=2, row_cts=2, page_rows=4, prompts=1, branches=2,
             lo=5, hi=7, rows=1),
        # Sixteen prompts, four branches each, K and V of a token as the outputs of the diagonal product at 2^13.
        dict(name="step-64-branches-n13", kind="step", log_n=13, limbs=2, row_cts=2, page_rows=16, prompts=16,
             branches=4, lo=60, hi=230, rows=1),
        # A few sequences end in a small cache.
        dict(name="compact-40-pages-n10", kind="compact", log_n=10, limbs=2, row_cts=2, page_rows=4, pages=40, seqs=9,
             lo=3, hi=17, freed=3),
        # A long-running cache of 4 GiB gives up its tail.
        dict(name="compact-1024-pages-n13", kind="compact", log_n=13, limbs=2, row_cts=2, page_rows=16, pages=1024,
             seqs=64, lo=40, hi=400, freed=20),
        # Rows of a few short sequences leave for the trusted side, and of many ragged ones.
        dict(name="gather-3-seqs-n11", kind="gather", log_n=11, limbs=3, row_cts=2, page_rows=4, seqs=3, lo=1, hi=9),
        dict(name="gather-48-seqs-n13", kind="gather", log_n=13, limbs=2, row_cts=2, page_rows=16, seqs=48, lo=1,
             hi=201),
        # The trusted side reads one short sequence, and a batch of long ones.
        dict(name="decrypt-1-seq-n10", kind="decrypt", log_n=10, limbs=2, row_cts=2, page_rows=4, seqs=1, lo=7, hi=7),
        dict(name="decrypt-32-seqs-n13", kind="decrypt", log_n=13, limbs=2, row_cts=2, page_rows=16, seqs=32, lo=1,
             hi=127),
    ]


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _draw_once(rng):
    kind = rng.choice(["q4", "q4", "q4", "step", "step", "compact", "gather", "decrypt"])
    if kind == "q4":
        return dict(kind=kind, log_n=rng.randint(10, 16), limbs=rng.randint(1, 8), log_scale=rng.randint(25, 28),
                    d_in=_spread(rng, 1, 4096), d_out=_spread(rng, 1, 4096),
                    group=rng.choice([32, 64, 96, 128, 256, 1024]), zeros=rng.random() < 0.5)
    c = dict(kind=kind, log_n=rng.randint(10, 16), limbs=rng.randint(1, 4), row_cts=rng.randint(1, 3),
             page_rows=rng.choice([1, 3, 4, 8, 16, 32]))
    lo = _spread(rng, 1, 100)
    hi = lo + _spread(rng, 1, 300)
    if kind == "step":
        c.update(prompts=_spread(rng, 1, 16), branches=rng.randint(1, 6), lo=lo, hi=hi, rows=_spread(rng, 1, 40))
    elif kind == "compact":
        seqs = _spread(rng, 2, 64)
        most = sum(-(-v // c["page_rows"]) for v in _lens(seqs, lo, hi))
        c.update(pages=round(most * rng.uniform(1.0, 1.5)), seqs=seqs, lo=lo, hi=hi, freed=rng.randint(1, seqs - 1))
    else:
        c.update(seqs=_spread(rng, 1, 64), lo=lo, hi=hi)
    return c


def draw(rng):
    while True:
        c = _draw_once(rng)
        w = work(c)
        # no larger than the largest listed case in memory, in traffic and in operations
        if w["bytes"] <= 2.4e9 and w["flops"] <= 1.8e12 and _state_bytes(c) <= 6e9:
            return c


def _lens(count, lo, hi):
    """Ragged lengths in [lo, hi], the same for every seed."""
    return [lo + (((i + 1) * 2654435761 % (1 << 32)) * (hi - lo + 1) >> 32) for i in range(count)]


def _row_words(c):
    return c["row_cts"] * 2 * c["limbs"] << c["log_n"]


def _pages_of(rows, page_rows):
    return -(-rows // page_rows)


def _step_counts(c):
    """Rows that every branch gets, and rows of its last page that are copied first."""
    lens = [v for v in _lens(c["prompts"], c["lo"], c["hi"]) for _ in range(c["branches"])]
    new = [1 + (i % c["rows"]) for i in range(len(lens))]
    return lens, new, [v % c["page_rows"] for v in lens]


def _live(c):
    """Pages that stay, and how many of them lie past the compacted end."""
    lens = _lens(c["seqs"], c["lo"], c["hi"])
    live = sum(_pages_of(v, c["page_rows"]) for v in lens[c["freed"]:])
    return live, round(live * (c["pages"] - live) / c["pages"])


def _state_bytes(c):
    if c["kind"] == "q4":
        words = 2 * c["limbs"] << c["log_n"]
        return 4 * words * (c["d_in"] + c["d_out"])
    pages = c["pages"] if c["kind"] == "compact" else _pool_pages(c)
    return 4 * pages * c["page_rows"] * _row_words(c)


def _pool_pages(c):
    p = c["page_rows"]
    if c["kind"] == "step":
        lens, new, _ = _step_counts(c)
        prompt = sum(_pages_of(v, p) for v in _lens(c["prompts"], c["lo"], c["hi"]))
        return prompt + sum(_pages_of(a + b, p) - a // p for a, b in zip(lens, new)) + 2
    return sum(_pages_of(v, p) for v in _lens(c["seqs"], c["lo"], c["hi"])) + 3


def work(case):
    n, L = 1 << case["log_n"], case["limbs"]
    if case["kind"] == "q4":
        d_in, d_out, groups = case["d_in"], case["d_out"], _pages_of(case["d_in"], case["group"])
        cols = 2 * L * n
        # flops: one modular multiply-add is counted as two, though a 30-bit residue takes four products of 8 bits
        return {"bytes": 4 * cols * (d_in + d_out) + d_out * (-(-d_in // 2)) + d_out * groups * (5 if case["zeros"] else 4),
                "flops": 2 * d_out * d_in * cols}
    row = 4 * _row_words(case)
    if case["kind"] == "step":
        _, new, copied = _step_counts(case)
        rows = sum(new) + sum(copied)
        return {"bytes": 2 * rows * row + 8 * rows, "flops": 0}
    if case["kind"] == "compact":
        return {"bytes": 2 * _live(case)[1] * case["page_rows"] * row + 8 * case["pages"], "flops": 0}
    rows = sum(_lens(case["seqs"], case["lo"], case["hi"]))
    if case["kind"] == "gather":
        return {"bytes": 2 * rows * row + 8 * rows, "flops": 0}
    # decrypt: a multiply-add and (log2 N) / 2 butterflies of a product, a sum and a difference a coefficient
    coeffs = rows * case["row_cts"] * L * n
    return {"bytes": rows * row * 3 // 2 + 4 * L * n + 8 * rows, "flops": coeffs * (2 + 3 * case["log_n"] // 2)}


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


@functools.lru_cache(maxsize=None)
def _inverse_roots(log_n, limbs):
    """(psi^-brv(k) as [L][N], N^-1 as [L]): psi the smallest primitive 2N-th root of unity."""
    n = 1 << log_n
    brv = np.zeros(n, dtype=np.int64)
    for b in range(log_n):
        brv |= ((np.arange(n) >> b) & 1) << (log_n - 1 - b)
    tables, ninv = [], []
    for q in _moduli(log_n, limbs):
        g = next(pow(x, (q - 1) // (2 * n), q) for x in range(2, q) if pow(x, (q - 1) // 2, q) == q - 1)
        odd = np.ones(1, dtype=np.int64) * g  # the odd powers of g, by doubling
        while odd.size < n:
            odd = np.concatenate([odd, odd * pow(g, 2 * odd.size, q) % q])
        inv = pow(int(odd.min()), -1, q)
        powers = np.ones(1, dtype=np.int64)
        while powers.size < n:
            powers = np.concatenate([powers, powers * pow(inv, powers.size, q) % q])
        tables.append(powers[brv])
        ninv.append(pow(n, -1, q))
    return np.stack(tables), np.array(ninv, dtype=np.int64)


# ---- inputs -----------------------------------------------------------------

def _residues(g, prefix, qs, n):
    """int32 residues prefix + (L, n), limb l uniform below qs[l]."""
    out = torch.empty(tuple(prefix) + (len(qs), n), dtype=torch.int32, device="cuda")
    for l, q in enumerate(qs):
        out[..., l, :] = torch.randint(0, q, tuple(prefix) + (n,), generator=g, device="cuda", dtype=torch.int32)
    return out


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, L = 1 << case["log_n"], case["limbs"]
    qs = _moduli(case["log_n"], L)
    st = {"case": case, "q": torch.tensor(qs, dtype=torch.int64, device="cuda").view(L, 1)}
    if own:
        import paper_2606_17421_amd as ck
        st["ck"] = ck
        st["ctx"] = ck.Context(case["log_n"], L)
    (_prepare_q4 if case["kind"] == "q4" else _prepare_cache)(case, seed, g, qs, n, st)
    return st


def _prepare_q4(case, seed, g, qs, n, st):
    d_in, d_out, group = case["d_in"], case["d_out"], case["group"]
    groups = _pages_of(d_in, group)
    w = torch.randn((d_out, groups * group), generator=g, device="cuda") * WEIGHT_STD
    w[:, d_in:] = 0
    w = w.view(d_out, groups, group)
    if case["zeros"]:
        low, high = w.amin(2), w.amax(2)
        scales = ((high - low) / 15).contiguous()
        zeros = torch.round(-low / scales).clamp_(0, 15)
    else:
        scales = (w.abs().amax(2) / 7).contiguous()
        zeros = torch.full_like(scales, 8)
    u = (torch.round(w / scales[:, :, None]) + zeros[:, :, None]).clamp_(0, 15).to(torch.uint8).view(d_out, -1)
    width = (d_in + 1) // 2
    u = torch.nn.functional.pad(u, (0, max(0, 2 * width - u.shape[1])))[:, :2 * width]
    if d_in % 2:
        u[:, d_in] = 0
    st["w4"] = (u[:, 0::2] | (u[:, 1::2] << 4)).contiguous()
    st["scales"] = scales
    st["zeros"] = zeros.to(torch.uint8) if case["zeros"] else None
    st["ct"] = _residues(g, (d_in, 2), qs, n)
    if own:
        ck, ctx, L = st["ck"], st["ctx"], case["limbs"]
        st["enc"] = ck.empty_workspace(ck.ckks_q4_weight_bytes(ctx, d_out, d_in, group, L, case["zeros"]))
        ck.ckks_linear_encode_q4(ctx, st["w4"], scales, st["zeros"], d_out, d_in, group, L,
                                 float(1 << case["log_scale"]), st["enc"])
        st["out"] = ck.empty_u32((d_out, 2, L, n))


def _prepare_cache(case, seed, g, qs, n, st):
    p, kind, host = case["page_rows"], case["kind"], np.random.default_rng(seed)
    branches = case["prompts"] * case["branches"] if kind == "step" else 0
    held = _lens(case["prompts"] if kind == "step" else case["seqs"], case["lo"], case["hi"])
    seqs = len(held) + branches
    pages = case["pages"] if kind == "compact" else _pool_pages(case)
    grown = max([a + b for a, b in zip(*_step_counts(case)[:2])]) if kind == "step" else 0
    max_pages = _pages_of(max(held + [grown]), p) + 1
    used = [_pages_of(v, p) for v in held]
    if kind == "compact":  # what stays is scattered over the pool, a set share of it past the compacted end
        live, above = _live(case)
        below = host.permutation(live)[: live - above]
        past = live + host.permutation(pages - live)[:above]
        stays = host.permutation(np.concatenate([below, past]))
        rest = host.permutation(np.setdiff1d(np.arange(pages), stays))
        order = np.concatenate([rest[: sum(used[: case["freed"]])], stays])
    else:
        order = host.permutation(pages)
    lens, refs = np.zeros(seqs, dtype=np.int32), np.zeros(pages, dtype=np.int32)
    table = np.full((seqs, max_pages), -1, dtype=np.int32)
    lens[: len(held)] = held
    at = 0
    for i, k in enumerate(used):
        table[i, :k] = order[at : at + k]
        refs[order[at : at + k]] = 1
        at += k
    st["lens"], st["refs"], st["table"] = _ints(lens), _ints(refs), _ints(table)
    rows_shape = (case["row_cts"], 2)
    st["pool"] = _residues(g, (pages, p) + rows_shape, qs, n)
    if kind == "step":
        old, new, _ = _step_counts(case)
        st["src"] = _ints(np.repeat(np.arange(case["prompts"]), case["branches"]))
        st["dst"] = _ints(np.arange(case["prompts"], seqs))
        st["row0"] = _ints(np.concatenate([[0], np.cumsum(new)]))
        st["rows"] = _residues(g, (sum(new),) + rows_shape, qs, n)
        st["status"] = torch.zeros(branches, dtype=torch.int32, device="cuda")
        # what a scheduler knows of its lengths on the host: request and place of every new and every copied row
        st["request"] = torch.from_numpy(np.repeat(np.arange(branches), new)).cuda()
        st["place"] = torch.from_numpy(np.concatenate([np.arange(a, a + b) for a, b in zip(old, new)])).cuda()
        part = [v % p for v in old]
        st["cow_request"] = torch.from_numpy(np.repeat(np.arange(branches), part)).cuda()
        st["cow_slot"] = torch.from_numpy(np.concatenate([np.arange(v) for v in part])).cuda()
        st["most_new"] = max(_pages_of(a + b, p) - a // p for a, b in zip(old, new))
    elif kind == "compact":
        st["lens0"], st["refs0"], st["table0"] = st["lens"].clone(), st["refs"].clone(), st["table"].clone()
        st["ended"] = _ints(np.arange(case["freed"]))
        st["live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    else:
        take = host.permutation(case["seqs"])
        st["seq"] = _ints(np.repeat(take, np.array(held)[take]))
        st["pos"] = _ints(np.concatenate([np.arange(held[i]) for i in take]))
    if kind == "decrypt":
        # the transform of a ternary secret is spread like uniform residues
        st["s"] = _residues(g, (), qs, n)
        tables, ninv = _inverse_roots(case["log_n"], case["limbs"])
        st["inv"] = torch.from_numpy(tables).cuda()
        st["ninv"] = torch.from_numpy(ninv).cuda().view(-1, 1)
    if own:
        ck, ctx = st["ck"], st["ctx"]
        st["cache"] = ck.Cache(ctx, st["pool"], st["refs"], st["table"], st["lens"])
        if kind == "step":
            need = ck.ckks_cache_workspace_bytes(ctx, st["cache"], ck.CKKS_CACHE_APPEND, branches, len(st["rows"]))
            st["ws"] = ck.empty_workspace(need)
        elif kind == "compact":
            st["ws"] = ck.empty_workspace(ck.ckks_cache_workspace_bytes(ctx, st["cache"], ck.CKKS_CACHE_COMPACT))
        else:
            shape = (len(st["seq"]), case["row_cts"]) + ((2,) if kind == "gather" else ()) + (case["limbs"], n)
            st["out"] = ck.empty_u32(shape)


# ---- one pass ---------------------------------------------------------------

def run(state):
    return _RUN[state["case"]["kind"]](state)


def _run_q4(st):
    c = st["case"]
    if own:
        st["ck"].ckks_linear_mac_q4(st["ctx"], st["enc"], st["ct"], st["out"], c["d_out"], c["d_in"], c["group"],
                                    c["limbs"], c["zeros"])
        return st["out"]
    d_in, d_out, L, q = c["d_in"], c["d_out"], c["limbs"], st["q"]
    u = torch.stack([st["w4"] & 15, st["w4"] >> 4], 2).view(d_out, -1)[:, :d_in].to(torch.int64)
    z = st["zeros"].to(torch.int64) if c["zeros"] else torch.full_like(st["scales"], 8, dtype=torch.int64)
    s = torch.round(st["scales"].double() * (1 << c["log_scale"])).to(torch.int64)
    of = torch.arange(d_in, device="cuda") // c["group"]
    w = ((u - z[:, of]) * s[:, of])[None].remainder(q[:, :, None])                   # [L][d_out][d_in]
    x = st["ct"].permute(2, 0, 1, 3).reshape(L, d_in, -1)                            # [L][d_in][2 N]
    # halves of 15 bits: every product of two matrices is exact in fp64 (2^30 d_in < 2^53)
    wh, wl = (w >> 15).double(), (w & 32767).double()
    xh, xl = (x >> 15).double(), (x & 32767).double()
    m = q[:, :, None]
    out = torch.bmm(wh, xh).to(torch.int64).remainder_(m).mul_(1 << 15)
    out += torch.bmm(wh, xl).add_(torch.bmm(wl, xh)).to(torch.int64)
    out = out.remainder_(m).mul_(1 << 15)
    out += torch.bmm(wl, xl).to(torch.int64)
    out = out.remainder_(m).to(torch.int32)
    return out.view(L, d_out, 2, -1).permute(1, 2, 0, 3).contiguous()


def _release(st, seq):
    """The sequences' pages lose a holder each; the sequences are left empty."""
    held = st["table"][seq].to(torch.int64)
    st["refs"].index_add_(0, held.clamp(min=0).view(-1), -(held >= 0).to(torch.int32).view(-1))
    st["table"][seq] = -1
    st["lens"][seq] = 0


def _run_step(st):
    c, p = st["case"], st["case"]["page_rows"]
    if own:
        ck = st["ck"]
        ck.ckks_cache_fork(st["ctx"], st["cache"], st["src"], st["dst"], st["status"])
        ck.ckks_cache_append(st["ctx"], st["cache"], st["dst"], st["row0"], st["rows"], st["ws"], st["status"])
        return {k: st[k] for k in ("pool", "refs", "table", "lens", "status")}
    src, dst = st["src"].to(torch.int64), st["dst"].to(torch.int64)
    refs, table, lens, pool = st["refs"], st["table"], st["lens"], st["pool"]
    # fork: the branches hold what their prompts hold
    _release(st, dst)
    table[dst] = table[src]
    lens[dst] = lens[src]
    held = table[dst].to(torch.int64)
    refs.index_add_(0, held.clamp(min=0).view(-1), (held >= 0).to(torch.int32).view(-1))
    # append: pages for what does not fit, and for a last page that others hold too
    old = lens[dst].to(torch.int64)
    new = (st["row0"][1:] - st["row0"][:-1]).to(torch.int64)
    first = old // p
    cow = old % p > 0                                     # the prompt holds it too
    start = torch.where(cow, first, (old + p - 1) // p)   # first position that gets a page
    need = (old + new + p - 1) // p - start
    base = torch.cumsum(need, 0) - need
    vacant = torch.argsort((refs != 0).to(torch.int32), stable=True)
    k = torch.arange(st["most_new"], device="cuda")[None, :]
    gets = k < need[:, None]
    page = vacant[(base[:, None] + k).clamp(max=len(vacant) - 1)]
    at = (start[:, None] + k).clamp(max=table.shape[1] - 1)
    before = torch.gather(table[dst].to(torch.int64), 1, first[:, None])[:, 0]
    held = table[dst].to(torch.int64)
    spare = torch.full((len(dst), 1), -1, dtype=torch.int64, device="cuda")
    held = torch.cat([held, spare], 1).scatter_(1, torch.where(gets, at, table.shape[1]), page)[:, :-1]
    table[dst] = held.to(torch.int32)
    refs.index_add_(0, before.clamp(min=0), -cow.to(torch.int32))
    refs.index_add_(0, page.view(-1), gets.to(torch.int32).view(-1))
    lens[dst] = (old + new).to(torch.int32)
    # the rows
    flat = pool.view(pool.shape[0] * p, -1)
    who, slot = st["cow_request"], st["cow_slot"]
    if len(who):
        now = torch.gather(held, 1, first[:, None].clamp(max=held.shape[1] - 1))[:, 0]
        flat[now[who] * p + slot] = flat[before[who] * p + slot]
    place = st["place"]
    flat[held[st["request"], place // p] * p + place % p] = st["rows"].view(len(place), -1)
    return {"pool": pool, "refs": refs, "table": table, "lens": lens, "status": torch.zeros_like(st["status"])}


def _run_compact(st):
    # the bookkeeping as it was before the sequences ended (pages that move leave their old place as it is)
    st["lens"].copy_(st["lens0"])
    st["refs"].copy_(st["refs0"])
    st["table"].copy_(st["table0"])
    if own:
        ck = st["ck"]
        ck.ckks_cache_free(st["ctx"], st["cache"], st["ended"])
        ck.ckks_cache_compact(st["ctx"], st["cache"], st["live"], st["ws"])
        return {k: st[k] for k in ("pool", "refs", "table", "lens", "live")}
    _release(st, st["ended"].to(torch.int64))
    refs, table, pool = st["refs"], st["table"], st["pool"]
    here = torch.arange(len(refs), device="cuda")
    full = refs > 0
    live = full.sum()
    moves = full & (here >= live)
    holes = ~full & (here < live)
    # the k-th page past the end goes to the k-th hole
    to = torch.argsort((~holes).to(torch.int32), stable=True)[(torch.cumsum(moves, 0) - 1).clamp(min=0)]
    count = _live(st["case"])[1]
    source = torch.argsort((~moves).to(torch.int32), stable=True)[:count]
    pool[to[source]] = pool[source]
    where = torch.where(moves, to, here)
    table.copy_(torch.where(table >= 0, where[table.to(torch.int64).clamp(min=0)].to(torch.int32), table))
    moved = torch.zeros_like(refs).index_add_(0, where, refs)
    refs.copy_(moved)
    return {"pool": pool, "refs": refs, "table": table, "lens": st["lens"], "live": live.to(torch.int32).view(1)}


def _taken(st):
    """The rows that (seq, pos) name, through the table."""
    p, pool = st["case"]["page_rows"], st["pool"]
    seq, pos = st["seq"].to(torch.int64), st["pos"].to(torch.int64)
    page = st["table"][seq, pos // p].to(torch.int64)
    return pool.view(-1, *pool.shape[2:])[page * p + pos % p]


def _run_gather(st):
    if own:
        st["ck"].ckks_cache_gather(st["ctx"], st["cache"], st["seq"], st["pos"], st["out"])
        return st["out"]
    return _taken(st)


def _run_decrypt(st):
    if own:
        st["ck"].ckks_cache_decrypt(st["ctx"], st["cache"], st["seq"], st["pos"], st["s"], st["out"])
        return st["out"]
    rows, q, n = _taken(st).to(torch.int64), st["q"], 1 << st["case"]["log_n"]
    a = (rows[:, :, 0] + rows[:, :, 1] * st["s"]) % q                                # [rows][row_cts][L][N]
    half, width = n // 2, 1
    while half:  # stage by stage: pairs at distance `width` give their sum, and their difference times a root
        v = a.view(*a.shape[:3], half, 2, width)
        tw = st["inv"][:, half : 2 * half, None]
        m = q[:, :, None]
        a = torch.stack([(v[..., 0, :] + v[..., 1, :]) % m, (v[..., 0, :] - v[..., 1, :] + m) * tw % m], 4)
        a = a.view(*rows.shape[:2], -1, n)
        half, width = half // 2, width * 2
    return (a * st["ninv"] % q).to(torch.int32)


_RUN = {"q4": _run_q4, "step": _run_step, "compact": _run_compact, "gather": _run_gather, "decrypt": _run_decrypt}


# ---- the definitions --------------------------------------------------------

def exact(case, seed):
    """From the definitions in 64-bit integers, entry by entry; None for cases that take too long."""
    w, n = work(case), 1 << case["log_n"]
    if own or w["bytes"] > 4e7 or w["flops"] > 4e8:
        return None
    if case["kind"] == "decrypt" and w["bytes"] * n > 4e9:  # a sum over N for every coefficient
        return None
    st = prepare(case, seed)
    q = np.array(_moduli(case["log_n"], case["limbs"]), dtype=np.int64)
    host = {k: v.cpu().numpy() for k, v in st.items() if isinstance(v, torch.Tensor)}
    return _EXACT[case["kind"]](case, host, q)


def _exact_q4(case, h, q):
    x = h["ct"].astype(np.int64)
    out = np.zeros((case["d_out"],) + x.shape[1:], dtype=np.int64)
    for j in range(case["d_out"]):
        for i in range(case["d_in"]):
            u = int(h["w4"][j, i // 2]) >> (4 * (i % 2)) & 15
            k = i // case["group"]
            z = int(h["zeros"][j, k]) if case["zeros"] else 8
            s = int(np.rint(np.float64(h["scales"][j, k]) * (1 << case["log_scale"])))
            weight = np.array([(u - z) * s % int(v) for v in q], dtype=np.int64)
            out[j] = (out[j] + weight[None, :, None] * x[i]) % q[None, :, None]
    return torch.from_numpy(out.astype(np.int32))


def _exact_free(h, s):
    for page in h["table"][s]:
        if page >= 0:
            h["refs"][page] -= 1
    h["table"][s], h["lens"][s] = -1, 0


def _exact_step(case, h, q):
    p = case["page_rows"]
    for src, dst in zip(h["src"], h["dst"]):
        _exact_free(h, dst)
        h["table"][dst], h["lens"][dst] = h["table"][src], h["lens"][src]
        for page in h["table"][dst]:
            if page >= 0:
                h["refs"][page] += 1
    for i, s in enumerate(h["dst"]):
        for r in range(h["row0"][i], h["row0"][i + 1]):
            at, slot = divmod(int(h["lens"][s]), p)
            page = h["table"][s, at] if slot else -1
            if page < 0 or h["refs"][page] > 1:
                fresh = int(np.flatnonzero(h["refs"] == 0)[0])
                if page >= 0:
                    h["pool"][fresh, :slot] = h["pool"][page, :slot]
                    h["refs"][page] -= 1
                h["refs"][fresh], h["table"][s, at], page = 1, fresh, fresh
            h["pool"][page, slot] = h["rows"][r]
            h["lens"][s] += 1
    return {k: torch.from_numpy(h[k]) for k in ("pool", "refs", "table", "lens")} | {
        "status": torch.zeros(len(h["dst"]), dtype=torch.int32)}


def _exact_compact(case, h, q):
    for s in h["ended"]:
        _exact_free(h, s)
    live = int((h["refs"] > 0).sum())
    for page in range(live, len(h["refs"])):
        if h["refs"][page] > 0:
            hole = int(np.flatnonzero(h["refs"] == 0)[0])
            h["pool"][hole] = h["pool"][page]
            h["refs"][hole], h["refs"][page] = h["refs"][page], 0
            h["table"][h["table"] == page] = hole
    return {k: torch.from_numpy(h[k]) for k in ("pool", "refs", "table", "lens")} | {
        "live": torch.tensor([live], dtype=torch.int32)}


def _exact_gather(case, h, q):
    p = case["page_rows"]
    rows = [h["pool"][h["table"][s, i // p], i % p] for s, i in zip(h["seq"], h["pos"])]
    return torch.from_numpy(np.stack(rows))


def _exact_decrypt(case, h, q):
    """m_k = N^-1 sum_i A_i psi^(-(2 brv(i) + 1) k), the sum written out."""
    log_n, n = case["log_n"], 1 << case["log_n"]
    rows = _exact_gather(case, h, q).numpy().astype(np.int64)
    out = np.zeros(rows.shape[:2] + rows.shape[3:], dtype=np.int32)
    odd = [2 * int(format(i, "0%db" % log_n)[::-1], 2) + 1 for i in range(n)]
    for l, m in enumerate(int(v) for v in q):
        inv = int(h["inv"][l, n // 2])  # psi^-brv(N/2) is psi^-1
        powers = np.ones(2 * n, dtype=np.int64)
        for k in range(1, 2 * n):
            powers[k] = powers[k - 1] * inv % m
        a = (rows[:, :, 0, l] + rows[:, :, 1, l] * h["s"][l].astype(np.int64)) % m
        total = np.zeros_like(a)
        k = np.arange(n, dtype=np.int64)
        for i in range(n):
            total = (total + a[..., i, None] * powers[odd[i] * k % (2 * n)]) % m
        out[:, :, l] = total * pow(n, -1, m) % m
    return torch.from_numpy(out)


_EXACT = {"q4": _exact_q4, "step": _exact_step, "compact": _exact_compact, "gather": _exact_gather,
          "decrypt": _exact_decrypt}
