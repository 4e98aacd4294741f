"""Calls of more workgroups than one launch has: a launch has fewer than 2^32 work-items, and the
declared ranges of requests, bundles and rings hold more.  Requests repeat a few pairs of expert and
bundle (sums a few lists of terms), so that every output is compared, on the device, with a small call's."""
import numpy as np
import pytest

from oracle import fp8 as OF
from test_gpu_experts import experts_of, ints
from test_gpu_fp8 import ctx_for
from workloads import gen

gpu = pytest.mark.gpu


def residues(ctx, *shape, seed=7):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.empty(shape + (ctx.limbs, ctx.n), dtype=torch.int32, device="cuda")
    for l, q in enumerate(ctx.moduli):
        t[..., l, :] = torch.randint(0, q, shape + (ctx.n,), generator=g, device="cuda", dtype=torch.int32)
    return t


def repeats(out, want):
    """Whether out[r] is want[r % len(want)] for every r, in pieces of up to 1 GiB."""
    k = len(want)
    step = max(1, (1 << 28) // want.numel()) * k
    for i in range(0, len(out), step):
        part = out[i:i + step]
        whole = len(part) // k * k
        if not bool((part[:whole].view(-1, *want.shape) == want).all()) or not bool((part[whole:] == want[:len(part) - whole]).all()):
            return False
    return True


def check_experts(ck, log_n, limbs, count, d_out, d_in):
    import torch
    ctx = ctx_for(ck, log_n, limbs)
    layers, enc = experts_of(ck, ctx, 900, 2, d_out, d_in, 128, limbs)
    ct = residues(ctx, 3, d_in, 2)
    pairs = [(0, 0), (1, 2), (1, 0), (0, 1), (0, 2)]
    want = ck.empty_u32((len(pairs), d_out, 2, limbs, ctx.n))
    expert, bundle = (ints([p[i] for p in pairs]) for i in range(2))
    ck.ckks_experts_mac_fp8(ctx, enc, expert, bundle, ct, want, d_out, d_in, limbs)
    cols = [0, 31, 32, 127, 128, ctx.n - 1]
    for k, (e, b) in enumerate(pairs):
        sample = ct[b][..., cols].cpu().numpy().view(np.uint32)
        assert np.array_equal(want[k][..., cols].cpu().numpy().view(np.uint32), OF.mac(*layers[e], sample, 128, 2.0 ** 30, ctx.moduli))
    out = ck.empty_u32((count, d_out, 2, limbs, ctx.n))
    out.fill_(-1)
    status = ints([7] * count)
    again = torch.arange(count, device="cuda") % len(pairs)
    ck.ckks_experts_mac_fp8(ctx, enc, expert[again], bundle[again], ct, out, d_out, d_in, limbs, status)
    assert not status.any()
    assert repeats(out, want)


@gpu
@pytest.mark.parametrize("d_out,d_in", [(1, 1), (9, 130), (5, 300)])
def test_experts_in_two_pieces(gpu_lib, d_out, d_in):
    check_experts(gpu_lib, 10, 16, 4099, d_out, d_in)


@gpu
@pytest.mark.parametrize("d_out,d_in", [(1, 1), (3, 130)])
def test_experts_in_two_pieces_without_a_list_of_bundles(gpu_lib, d_out, d_in):
    """A request has the bundle of its own number, in the second piece as well; the last two have none."""
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 16)
    _, enc = experts_of(ck, ctx, 905, 2, d_out, d_in, 128, 16)
    count, bundles = 4101, 4099
    few = residues(ctx, 6, d_in, 2)
    again = torch.arange(bundles, device="cuda") % 6
    expert = (torch.arange(count, device="cuda") % 2).to(torch.int32)
    want = ck.empty_u32((6, d_out, 2, 16, ctx.n))
    ck.ckks_experts_mac_fp8(ctx, enc, expert[:6].contiguous(), None, few, want, d_out, d_in, 16)
    out, status = ck.empty_u32((count, d_out, 2, 16, ctx.n)), ints([7] * count)
    out.fill_(-5)
    ck.ckks_experts_mac_fp8(ctx, enc, expert, None, few[again], out, d_out, d_in, 16, status)
    assert not status[:bundles].any() and status[bundles:].tolist() == [1, 1]
    assert repeats(out[:bundles], want) and bool((out[bundles:] == -5).all())


@gpu
@pytest.mark.parametrize("d_in", [1, 130])
def test_experts_past_2_32_work_items(gpu_lib, d_in):
    """8 GiB of outputs: 2051 requests of 8 limbs of 2^16 coefficients, one output each."""
    check_experts(gpu_lib, 16, 8, 2051, 1, d_in)


def check_sums(ck, log_n, limbs, bundles, features):
    import torch
    ctx = ctx_for(ck, log_n, limbs)
    gates, y = residues(ctx, 3), residues(ctx, 3, features, 2, seed=8)
    lists = [[0, 1], [2, -1], [1, 1], [-1, -1], [2, 0]]
    want = ck.empty_u32((len(lists), features, 2, limbs, ctx.n))
    ck.ckks_experts_combine(ctx, gates, y, ints(lists), want, features, limbs)
    cols = [0, 1023, ctx.n - 1]
    pick = lambda t: t[..., cols].cpu().numpy().view(np.uint32)  # noqa: E731
    assert np.array_equal(pick(want), OF.combine(pick(gates), pick(y), lists, ctx.moduli).astype(np.uint32))
    out = ck.empty_u32((bundles, features, 2, limbs, ctx.n))
    out.fill_(-1)
    terms = ints(lists)[torch.arange(bundles, device="cuda") % len(lists)].contiguous()
    ck.ckks_experts_combine(ctx, gates, y, terms, out, features, limbs)
    assert repeats(out, want)


def room_for(gib):
    import torch
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of device memory")


@gpu
def test_sums_in_two_pieces(gpu_lib):
    check_sums(gpu_lib, 11, 16, 33001, 1)


@gpu
def test_sums_past_2_32_work_items(gpu_lib):
    """128 GiB of outputs: 32771 bundles of one feature, 8 limbs of 2^16 coefficients."""
    import torch
    room_for(150)
    check_sums(gpu_lib, 16, 8, 32771, 1)
    torch.cuda.empty_cache()


def check_encode(ck, log_n, limbs, d_out, d_in, block_rows, seed=930):
    """Layers whose rows repeat every 32: the encoding of a row tile is that of a layer of 32 rows."""
    import torch
    ctx = ctx_for(ck, log_n, limbs)
    g = torch.Generator(device="cuda").manual_seed(seed)
    part = torch.randint(0, 256, (32, d_in), generator=g, device="cuda", dtype=torch.uint8)
    part[(part & 127) == 127] = 3
    blocks, tiles, steps = -(-d_in // 128), -(-d_out // 32), -(-d_in // 32)
    scales = torch.randn((1, blocks), generator=g, device="cuda") * 2e-4
    w8 = torch.empty((d_out, d_in), dtype=torch.uint8, device="cuda")
    whole = d_out // 32 * 32
    w8[:whole].view(-1, 32, d_in).copy_(part)
    w8[whole:] = part[:d_out - whole]
    bad = ints([5])
    rows = -(-d_out // block_rows)
    enc = torch.empty(ck.ckks_fp8_weight_bytes(ctx, d_out, d_in, limbs), dtype=torch.uint8, device="cuda")
    enc.fill_(0xEE)
    ck.ckks_linear_encode_fp8(ctx, w8, scales.expand(rows, blocks).contiguous(), d_out, d_in, block_rows, limbs, 2.0 ** 30, enc, bad)
    assert int(bad) == 0
    del w8
    one = torch.empty(ck.ckks_fp8_weight_bytes(ctx, 32, d_in, limbs), dtype=torch.uint8, device="cuda")
    ck.ckks_linear_encode_fp8(ctx, part, scales, 32, d_in, 32, limbs, 2.0 ** 30, one)
    frag, sc = steps * 2048, blocks * 3 * 32 * 4
    full = d_out // 32
    assert repeats(enc[:full * frag].view(full, -1), one[:frag].view(1, -1))
    at = enc[tiles * frag:].view(limbs, tiles, sc)
    for l in range(limbs):
        assert repeats(at[l, :full], one[frag:].view(limbs, 1, sc)[l])


@gpu
@pytest.mark.parametrize("limbs,d_out,d_in", [(1, 16416, 16400), (16, 2080, 16400)])
def test_encode_fp8_in_pieces(gpu_lib, limbs, d_out, d_in):
    check_encode(gpu_lib, 10, limbs, d_out, d_in, 128)


@gpu
def test_encode_fp8_scales_past_2_32_work_items(gpu_lib):
    """16 limbs of 2^16 inputs and as many outputs as there may be: 32 GiB of weights, 112 GiB encoded."""
    import torch
    room_for(170)
    check_encode(gpu_lib, 10, 16, 524256, (1 << 16) + 128, 524256)
    torch.cuda.empty_cache()


@gpu
@pytest.mark.parametrize("d_out,d_in,rows", [(16416, 16400, 7), (65536 + 32, 65536, 11)])
def test_encode_scalar_past_a_launch(gpu_lib, d_out, d_in, rows):
    """More weights than a launch of 2^20 workgroups has, and than 2^32."""
    import torch
    ck = gpu_lib
    room_for(60)
    ctx = ctx_for(ck, 10, 1)
    g = torch.Generator(device="cuda").manual_seed(940)
    part = torch.randn((rows, d_in), generator=g, device="cuda", dtype=torch.float64)
    w = torch.empty((d_out, d_in), dtype=torch.float64, device="cuda")
    for r in range(rows):
        w[r::rows] = part[r]
    enc = torch.full((d_out, d_in), -1, dtype=torch.int32, device="cuda")
    ck.ckks_linear_encode_scalar(ctx, w, d_out, d_in, 1, 2.0 ** 26, enc)
    del w
    q = ctx.moduli[0]
    want = torch.round(part * 2.0 ** 26).to(torch.int64).remainder(q).to(torch.int32)
    assert repeats(enc, want)
    torch.cuda.empty_cache()


@gpu
@pytest.mark.parametrize("rows", [66003, (1 << 20) + 5])
def test_automorphism_past_a_launch(gpu_lib, rows):
    import torch
    ck = gpu_lib
    log_n = 12
    room_for(40)
    ctx = ctx_for(ck, log_n, 1)
    part = residues(ctx, 5)[:, 0].contiguous()
    want = torch.empty_like(part)
    ck.ckks_automorphism(ctx, part, 5, 5, want)
    src = part[torch.arange(rows, device="cuda") % 5]
    out = torch.full_like(src, -1)
    ck.ckks_automorphism(ctx, src, rows, 5, out)
    assert repeats(out, want)
    del src, out
    torch.cuda.empty_cache()


@gpu
@pytest.mark.parametrize("count", [16411, 1048583])
def test_add_past_a_launch(gpu_lib, count):
    """In place, 16 words of each coefficient a ciphertext: up to 128 GiB."""
    import torch
    ck = gpu_lib
    room_for(150 if count > 1 << 20 else 8)
    ctx = ctx_for(ck, 11, 8)
    part = residues(ctx, 3, 2)
    want = torch.empty_like(part)
    ck.ckks_add(ctx, part, part, 3, 8, want)
    a = ck.empty_u32((count, 2, 8, ctx.n))
    for r in range(3):
        a[r::3] = part[r]
    ck.ckks_add(ctx, a, a, count, 8, a)
    assert repeats(a, want)
    del a
    torch.cuda.empty_cache()


@gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("limbs,d_out,d_in", [(16, 4128, 8224), (16, 524256, (1 << 14) + 32)])
def test_encode_q4_past_a_launch(gpu_lib, limbs, d_out, d_in, zeros):
    import torch
    ck = gpu_lib
    room_for(60 if d_out > 1 << 16 else 8)
    ctx = ctx_for(ck, 10, 16)
    g = torch.Generator(device="cuda").manual_seed(950)
    groups, tiles = d_in // 32, d_out // 32
    part = torch.randint(0, 256, (32, d_in // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randn((32, groups), generator=g, device="cuda") * 1e-3
    zero = torch.randint(0, 16, (32, groups), generator=g, device="cuda", dtype=torch.uint8) if zeros else None

    def many(t):
        return None if t is None else t.expand(tiles, *t.shape).reshape(d_out, -1).contiguous()

    def encode(w, s, z, rows):
        enc = torch.full((ck.ckks_q4_weight_bytes(ctx, rows, d_in, 32, limbs, zeros),), 0xEE, dtype=torch.uint8, device="cuda")
        ck.ckks_linear_encode_q4(ctx, w, s, z, rows, d_in, 32, limbs, 2.0 ** 30, enc)
        return enc
    two = lambda t: None if t is None else torch.cat([t, t])  # noqa: E731
    one = encode(two(part), two(scales), two(zero), 64)     # rows are padded to 64
    enc = encode(many(part), many(scales), many(zero), d_out)
    frag, sc = groups * 64 * (16 if zeros else 8), groups * 32 * 8
    assert repeats(enc[:tiles * frag].view(tiles, -1), one[:frag].view(1, -1))
    padded = -(-tiles // 2) * 2
    at, small = enc[padded * frag:].view(limbs, padded, sc), one[2 * frag:].view(limbs, 2, sc)
    for l in range(limbs):
        assert repeats(at[l, :tiles], small[l, :1])
    del enc
    torch.cuda.empty_cache()


@gpu
@pytest.mark.parametrize("count,limbs", [((1 << 20) + 7, 1), (300000, 2), ((1 << 24) + 3, 1)])
def test_gather_past_a_launch(gpu_lib, count, limbs):
    """Rows of 8 and of 16 KiB, a few over and over, one of them absent: up to 128 GiB."""
    import torch
    ck = gpu_lib
    room_for(150 if count > 1 << 23 else 12)
    ctx = ctx_for(ck, 10, limbs)
    cache = ck.Cache.empty(ctx, 3, 2, 1, limbs, 1, 3)
    rows = residues(ctx, 5, 1, 2)
    ws = ck.empty_workspace(ck.ckks_cache_workspace_bytes(ctx, cache, ck.CKKS_CACHE_APPEND, 1, 5))
    ck.ckks_cache_append(ctx, cache, ints([0]), ints([0, 5]), rows, ws)
    at = ints([0, 3, 4, 9, 1, 2])
    want = torch.zeros((6, *rows.shape[1:]), dtype=torch.int32, device="cuda")
    for k, p in enumerate(at.tolist()):
        if p < 5:
            want[k] = rows[p]
    pos = at[torch.arange(count, device="cuda") % 6].contiguous()
    out = ck.empty_u32((count, *rows.shape[1:]))
    out.fill_(-1)
    ck.ckks_cache_gather(ctx, cache, torch.zeros_like(pos), pos, out)
    assert repeats(out, want)
    del out
    torch.cuda.empty_cache()


@gpu
def test_bsgs_of_many_inputs(gpu_lib):
    """Enough inputs that the giant steps' sums, four lanes a word, pass 2^32 work-items."""
    import torch
    ck = gpu_lib
    room_for(60)
    ctx = ctx_for(ck, 10, 3)
    count, n1, n2 = 174763 + 5, 1, 2
    pt, part = residues(ctx, n1 * n2)[:, :2].contiguous(), residues(ctx, 5, 2, seed=961)[:, :, :2].contiguous()
    ksk = residues(ctx, 1, 2, 2, seed=962)

    def product(ct, n):
        ws = ck.empty_workspace(ck.bsgs_workspace_bytes(ctx, n, n1, n2))
        out = torch.full((n, 2, 1, ctx.n), -1, dtype=torch.int32, device="cuda")
        ck.ckks_linear_bsgs(ctx, pt, ct, n, n1, n2, ksk, ws, out)
        return out
    want = product(part, 5)
    ct = part[torch.arange(count, device="cuda") % 5]
    assert repeats(product(ct, count), want)
    torch.cuda.empty_cache()


@gpu
def test_keys_past_a_launch(gpu_lib):
    import torch
    ck = gpu_lib
    room_for(24)
    ctx = ctx_for(ck, 10, 3)
    keys, half = 174763 + 4, ctx.n // 2
    s, a, e = residues(ctx), residues(ctx, 4, 2), torch.randint(-19, 20, (4, 2, ctx.n), dtype=torch.int32, device="cuda")
    many = torch.arange(keys, device="cuda") % 4

    def keygen(a, e, n):
        out = torch.full((n, 2, 2, 3, ctx.n), -1, dtype=torch.int32, device="cuda")
        ck.ckks_keygen_rotation(ctx, s, 3, half // 2, n, a, e, out)   # rotations by 3 and 3 + N/4 in turn
        return out
    want = keygen(a, e, 4)
    assert repeats(keygen(a[many], e[many], keys), want)
    torch.cuda.empty_cache()


@gpu
def test_more_rows_than_a_launch_are_refused(gpu_lib):
    """256 GiB of rows of 2^10, named by a buffer of a few: the sizes alone are looked at."""
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 3)
    some = ck.empty_u32((4, 2, 3, ctx.n))
    p, lib, rows = some.data_ptr(), ck._lib, 1 << 26
    cache = ck.Cache.empty(ctx, 1, 1, 1, 3, 1, 1)
    bad = ck.CKKS_E_INVALID_ARG
    import ctypes
    for call in (lambda: lib.ckks_ntt(ctx.handle, p, rows, 1, None), lambda: lib.ckks_intt(ctx.handle, p, rows // 2, 2, None),
                 lambda: lib.ckks_linear_encode_poly(ctx.handle, p, rows, 1, 1.0, p, None),
                 lambda: lib.ckks_encrypt(ctx.handle, None, p, p, p, rows, 1, p, None),
                 lambda: lib.ckks_decrypt(ctx.handle, p, p, rows, 1, p, None),
                 lambda: lib.ckks_cache_decrypt(ctx.handle, ctypes.byref(cache.struct), p, p, p, rows, p, None)):
        assert call() == bad
        assert "too many polynomials" in ck.ckks_last_error()
    assert lib.ckks_linear_bsgs(ctx.handle, p, p, 1 << 23, 1, 1, None, None, 0, p, None) == bad
    assert "count" in ck.ckks_last_error()
