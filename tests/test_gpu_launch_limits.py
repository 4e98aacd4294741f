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
