"""GPU parity of the experts' layers and of the gated sum of their outputs against
the oracle, bit for bit: ragged requests, bundles that several experts share,
requests that name nothing, captured calls, and the refusals."""
import numpy as np
import pytest

from oracle import fp8 as OF
from test_gpu_fp8 import ctx_for, encode, layer
from workloads import gen

gpu = pytest.mark.gpu


def experts_of(ck, ctx, seed, experts, d_out, d_in, block_rows, limbs, scale=2.0 ** 30):
    """Their layers, and their encoded weights one after the other."""
    import torch
    layers = [layer(seed + e, d_out, d_in, block_rows) for e in range(experts)]
    return layers, torch.stack([encode(ck, ctx, c, s, block_rows, limbs, scale) for c, s in layers])


def ints(a):
    import torch
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def check(ck, log_n, limbs, experts, expert, bundle, bundles, d_out, d_in, seed, block_rows=128):
    ctx = ctx_for(ck, log_n, limbs)
    layers, enc = experts_of(ck, ctx, seed, experts, d_out, d_in, block_rows, limbs)
    ct = gen.uniform_residues(np.random.default_rng(seed + 99), (bundles, d_in, 2), ctx.moduli, ctx.n)
    out = ck.empty_u32((len(expert), d_out, 2, limbs, ctx.n))
    out.fill_(-3)
    status = ints([7] * len(expert))
    ck.ckks_experts_mac_fp8(ctx, enc, ints(expert), None if bundle is None else ints(bundle), ck.to_device(ct), out, d_out, d_in,
                            limbs, status)
    got = ck.to_host_u32(out)
    named = list(range(len(expert))) if bundle is None else bundle
    cols = list(range(ctx.n)) if ctx.n <= 1024 and d_out * d_in <= 3000 else [0, 31, 32, 511, ctx.n - 1]
    for r, (e, b) in enumerate(zip(expert, named)):
        good = 0 <= e < experts and 0 <= b < bundles
        assert int(status[r]) == (ck.CKKS_EXPERT_OK if good else ck.CKKS_EXPERT_BAD_REQUEST)
        if good:
            want = OF.mac(*layers[e], ct[b][..., cols], block_rows, 2.0 ** 30, ctx.moduli).astype(np.uint32)
            assert np.array_equal(got[r][..., cols], want), r
        else:
            assert np.all(got[r].view(np.int32) == -3)


@gpu
@pytest.mark.parametrize("d_out,d_in", [(1, 1), (32, 32), (33, 40), (65, 129), (200, 300), (300, 100)])
def test_ragged_requests(gpu_lib, d_out, d_in):
    """An expert without requests, one with most of them, in no order; bundles that two experts share and one of none."""
    check(gpu_lib, 10, 2, 4, [0, 3, 3, 3, 1, 3, 0], [2, 2, 0, 1, 4, 4, 4], 5, d_out, d_in, 600)


@gpu
@pytest.mark.parametrize("d_out,d_in", [(20, 50), (290, 600), (70, 1100), (300, 1030)])
def test_many_columns(gpu_lib, d_out, d_in):
    check(gpu_lib, 11, 4, 3, [0, 0, 1, 2, 2], [0, 1, 1, 0, 2], 3, d_out, d_in, 620, 1)


@gpu
@pytest.mark.parametrize("d_out,d_in", [(5, 5), (40, 70), (130, 1300), (290, 1500), (300, 200), (270, 400), (300, 900), (290, 1200)])
def test_requests_that_name_nothing(gpu_lib, d_out, d_in):
    """At the ends and between good ones, and in every kernel of the layer."""
    big, small = 2 ** 31 - 1, -(2 ** 31)
    check(gpu_lib, 11, 4, 2, [-1, 0, 2, 1, big, small, 1, 0], [0, -1, 0, 1, 0, 0, 2, big], 2, d_out, d_in, 640)
    check(gpu_lib, 10, 1, 1, [-1], [0], 1, d_out, d_in, 641)


@gpu
def test_a_request_has_the_bundle_of_its_number(gpu_lib):
    check(gpu_lib, 10, 2, 3, [2, 0, 1, 0], None, 3, 33, 65, 650)


@gpu
def test_one_request_is_the_layer(gpu_lib):
    """The same words as ckks_linear_mac_fp8, for sizes of each of its kernels."""
    ck = gpu_lib
    for log_n, limbs, d_out, d_in in [(10, 1, 16, 16), (12, 4, 16, 1024), (12, 4, 300, 700), (12, 4, 300, 1500), (10, 1, 600, 70)]:
        ctx = ctx_for(ck, log_n, limbs)
        _, enc = experts_of(ck, ctx, 660, 2, d_out, d_in, 128, limbs)
        ct = ck.to_device(gen.uniform_residues(np.random.default_rng(661), (1, d_in, 2), ctx.moduli, ctx.n))
        a, b = ck.empty_u32((1, d_out, 2, limbs, ctx.n)), ck.empty_u32((d_out, 2, limbs, ctx.n))
        ck.ckks_experts_mac_fp8(ctx, enc, ints([1]), ints([0]), ct, a, d_out, d_in, limbs)
        ck.ckks_linear_mac_fp8(ctx, enc[1], ct[0], b, d_out, d_in, limbs)
        assert bool((a[0] == b).all()), (d_out, d_in)


@gpu
def test_empty_requests(gpu_lib):
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    out = ck.empty_u32((3, 4, 2, 2, ctx.n))
    out.fill_(5)
    status = ints([9, 9, 9])
    enc = ck.empty_workspace(2 * ck.ckks_fp8_weight_bytes(ctx, 4, 8, 2)).view(2, -1)
    ct = ck.empty_u32((2, 8, 2, 2, ctx.n))
    ck.ckks_experts_mac_fp8(ctx, enc, ints([]), ints([]), ct, out, 4, 8, 2)                      # no requests
    ck.ckks_experts_mac_fp8(ctx, enc[:0], ints([0, 1, 0]), ints([0, 0, 0]), ct, out, 4, 8, 2, status)   # no experts
    assert status.tolist() == [1, 1, 1] and np.all(ck.to_host_u32(out) == 5)
    ck.ckks_experts_mac_fp8(ctx, enc, ints([0, 1, 2]), ints([0, 0, 0]), ct, out, 0, 8, 2, status)       # no outputs
    assert status.tolist() == [0, 0, 1] and np.all(ck.to_host_u32(out) == 5)
    ck.ckks_experts_mac_fp8(ctx, enc, ints([0, -1, 1]), ints([0, 0, 1]), ct, out, 4, 0, 2, status)      # no inputs
    assert status.tolist() == [0, 1, 0]
    got = ck.to_host_u32(out)
    assert not got[[0, 2]].any() and np.all(got[1] == 5)


@gpu
def test_graphs_with_room(gpu_lib):
    """Two captured calls over one set of weights, replayed with lists that change and eager work between."""
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    d_out, d_in, experts, bundles, room = 40, 150, 3, 2, 4
    layers, enc = experts_of(ck, ctx, 670, experts, d_out, d_in, 128, 2)
    ct = gen.uniform_residues(np.random.default_rng(671), (bundles, d_in, 2), ctx.moduli, ctx.n)
    d_ct = ck.to_device(ct)
    want = {(e, b): OF.mac(*layers[e], ct[b], 128, 2.0 ** 30, ctx.moduli).astype(np.uint32) for e in range(experts) for b in range(bundles)}
    lists = [(ints([-1] * room), ints([0] * room), ck.empty_u32((room, d_out, 2, 2, ctx.n)), ints([0] * room)) for _ in range(2)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    for e, b, out, status in lists:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ck.ckks_experts_mac_fp8(ctx, enc, e, b, d_ct, out, d_out, d_in, 2, status, stream=s)
        graphs.append(g)
    for step, (es, bs) in enumerate([([0, 1, 2, -1], [0, 1, 1, 0]), ([2, 2, -1, -1], [0, 1, 0, 0]), ([-1] * 4, [0] * 4), ([1] * 4, [0, 1, 0, 1])]):
        for k, (e, b, out, status) in enumerate(lists):
            e.copy_(ints(es[::-1] if k else es))
            b.copy_(ints(bs[::-1] if k else bs))
            out.fill_(step)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for k, (_, _, out, status) in enumerate(lists):
            got = ck.to_host_u32(out)
            for r, (e, b) in enumerate(list(zip(es, bs))[::-1] if k else zip(es, bs)):
                assert int(status[r]) == (0 if e >= 0 else 1)
                assert np.array_equal(got[r], want[e, b]) if e >= 0 else np.all(got[r] == step)
    del graphs


@gpu
@pytest.mark.parametrize("top", [1, 2, 3, 4, 5, 6, 7, 8, 9, 15, 16, 17, 40])
@pytest.mark.parametrize("log_n,limbs,features", [(10, 2, 3), (12, 3, 1)])
def test_combine(gpu_lib, log_n, limbs, features, top):
    """Any number of terms a bundle, requests named twice, terms that name nothing, and a bundle of none."""
    ck = gpu_lib
    ctx = ctx_for(ck, log_n, limbs)
    rng = np.random.default_rng(700 + top)
    count, bundles = 5, 4
    gates = gen.uniform_residues(rng, (count,), ctx.moduli, ctx.n)
    y = gen.uniform_residues(rng, (count, features, 2), ctx.moduli, ctx.n)
    terms = rng.integers(-2, count + 2, (bundles, top))
    terms[0] = np.arange(top) % count          # all of them
    terms[1] = [-1] * top
    terms[2, 0] = 2 ** 31 - 1
    out = ck.empty_u32((bundles, features, 2, limbs, ctx.n))
    out.fill_(-1)
    ck.ckks_experts_combine(ctx, ck.to_device(gates), ck.to_device(y), ints(terms.tolist()), out, features, limbs)
    got = ck.to_host_u32(out)
    assert np.array_equal(got, OF.combine(gates, y, terms, ctx.moduli).astype(np.uint32))
    assert not got[1].any()


@gpu
@pytest.mark.parametrize("top", [1, 8, 15, 16, 31, 300])
def test_the_largest_gated_sums(gpu_lib, top):
    """Every residue q - 1, one request in all terms."""
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    ends = np.broadcast_to(np.array(ctx.moduli, np.uint32)[:, None] - 1, (2, ctx.n))
    gates, y = ends[None].copy(), np.broadcast_to(ends, (1, 2, 2) + ends.shape).copy()
    out = ck.empty_u32((1, 2, 2, 2, ctx.n))
    ck.ckks_experts_combine(ctx, ck.to_device(gates), ck.to_device(y), ints([[0] * top]), out, 2, 2)
    want = np.array([top % q for q in ctx.moduli], np.uint32)      # (q - 1)^2 is 1
    assert np.all(ck.to_host_u32(out) == want[:, None])


@gpu
@pytest.mark.parametrize("features", [1, 37, 700])
def test_combine_in_a_graph(gpu_lib, features):
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 11, 2)
    rng = np.random.default_rng(720)
    gates, y = gen.uniform_residues(rng, (4,), ctx.moduli, ctx.n), gen.uniform_residues(rng, (4, features, 2), ctx.moduli, ctx.n)
    d_g, d_y, terms = ck.to_device(gates), ck.to_device(y), ints([[0, 1], [3, -1], [2, 2]])
    out = ck.empty_u32((3, features, 2, 2, ctx.n))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        ck.ckks_experts_combine(ctx, d_g, d_y, terms, out, features, 2, stream=s)
    for lists in ([[0, 1], [3, -1], [2, 2]], [[-1, -1], [0, 3], [1, 2]]):
        terms.copy_(ints(lists))
        out.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(ck.to_host_u32(out), OF.combine(gates, y, lists, ctx.moduli).astype(np.uint32))
    del graph


@gpu
def test_combine_past_32_bits(gpu_lib):
    """Requests of 2 GiB: offsets of inputs and outputs pass 2^32 bytes; checked on a sample."""
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 16, 8)
    count, features = 3, 520
    g = torch.Generator(device="cuda").manual_seed(6)

    def residues(*shape):
        t = torch.empty(shape + (8, ctx.n), dtype=torch.int32, device="cuda")
        for l, q in enumerate(ctx.moduli):
            t[..., l, :] = torch.randint(0, q, shape + (ctx.n,), generator=g, device="cuda", dtype=torch.int32)
        return t
    gates, y = residues(count), residues(count, features, 2)
    out = ck.empty_u32((3, features, 2, 8, ctx.n))
    lists = [[2, 1], [0, -1], [2, 2]]
    ck.ckks_experts_combine(ctx, gates, y, ints(lists), out, features, 8)
    cols = torch.tensor([0, 1023, 1024, 40000, 65535], device="cuda")
    rows = torch.tensor([0, 1, 511, 512, 519], device="cuda")
    pick = lambda t: t[..., cols].cpu().numpy().view(np.uint32)  # noqa: E731
    assert np.array_equal(pick(out[:, rows]), OF.combine(pick(gates), pick(y[:, rows]), lists, ctx.moduli).astype(np.uint32))


@gpu
def test_empty_sums(gpu_lib):
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    gates, y, out = ck.empty_u32((2, 2, ctx.n)), ck.empty_u32((2, 3, 2, 2, ctx.n)), ck.empty_u32((2, 3, 2, 2, ctx.n))
    out.fill_(4)
    ck.ckks_experts_combine(ctx, gates, y, ints([]).view(0, 2), out, 3, 2)
    ck.ckks_experts_combine(ctx, gates, y, ints([[0], [1]]), out, 0, 2)
    assert np.all(ck.to_host_u32(out) == 4)
    ck.ckks_experts_combine(ctx, gates, y, torch.empty((2, 0), dtype=torch.int32, device="cuda"), out, 3, 2)
    assert not ck.to_host_u32(out).any()
    out.fill_(4)
    ck.ckks_experts_combine(ctx, gates[:0], y[:0], ints([[0], [1]]), out, 3, 2)
    assert not ck.to_host_u32(out).any()


@gpu
def test_refusals(gpu_lib):
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    d_out, d_in, bad = 16, 64, ck.CKKS_E_INVALID_ARG
    need = ck.ckks_fp8_weight_bytes(ctx, d_out, d_in, 2)
    enc = ck.empty_workspace(2 * need).view(2, -1)
    ct, out = ck.empty_u32((2, d_in, 2, 2, ctx.n)), ck.empty_u32((3, d_out, 2, 2, ctx.n))
    e, b, status = ints([0, 1, 1]), ints([0, 1, 0]), ints([0, 0, 0])
    raw = ck._lib.ckks_experts_mac_fp8

    def call(w=enc.data_ptr(), experts=2, ep=e.data_ptr(), bp=b.data_ptr(), count=3, x=ct.data_ptr(), bundles=2, y=out.data_ptr(),
             o=d_out, i=d_in, limbs=2, st=status.data_ptr()):
        return raw(ctx.handle, w, experts, ep, bp, count, x, bundles, y, o, i, limbs, st, None)
    for wrong in (dict(limbs=0), dict(limbs=3), dict(experts=65537), dict(count=65537), dict(bundles=65537), dict(o=524281),
                  dict(i=(1 << 24) + 1), dict(w=None), dict(ep=None), dict(x=None), dict(y=None), dict(w=enc.data_ptr() + 4),
                  dict(ep=e.data_ptr() + 2), dict(bp=b.data_ptr() + 1), dict(x=ct.data_ptr() + 4), dict(y=out.data_ptr() + 8),
                  dict(st=status.data_ptr() + 2), dict(y=ct.data_ptr()), dict(y=enc.data_ptr()), dict(st=e.data_ptr()),
                  dict(st=b.data_ptr()), dict(st=out.data_ptr()), dict(st=ct.data_ptr())):
        assert call(**wrong) == bad, wrong
        assert ck.ckks_last_error()
    with pytest.raises(ValueError):
        ck.ckks_experts_mac_fp8(ctx, enc, e.to(torch.int64), b, ct, out, d_out, d_in, 2)
    with pytest.raises(ValueError):
        ck.ckks_experts_mac_fp8(ctx, enc, e.float(), b, ct, out, d_out, d_in, 2)
    with pytest.raises(ValueError):
        ck.ckks_experts_mac_fp8(ctx, enc, e, b[:2], ct, out, d_out, d_in, 2)
    with pytest.raises(ValueError):
        ck.ckks_experts_mac_fp8(ctx, enc, e, b, ct, out[:2], d_out, d_in, 2)
    with pytest.raises(ValueError):   # weights of other sizes
        ck.ckks_experts_mac_fp8(ctx, enc, e, b, ct, out, d_out // 2, d_in // 2, 2)
    with pytest.raises(ValueError):
        ck.ckks_experts_mac_fp8(ctx, enc, e, b, ct, out, d_out, d_in, 2, status[:1])
    gates, y, terms = ck.empty_u32((3, 2, ctx.n)), out, ints([[0, 1], [2, -1]])
    to = ck.empty_u32((2, d_out, 2, 2, ctx.n))
    raw = ck._lib.ckks_experts_combine

    def total(g=gates.data_ptr(), x=y.data_ptr(), count=3, tp=terms.data_ptr(), bundles=2, top=2, z=to.data_ptr(), features=d_out, limbs=2):
        return raw(ctx.handle, g, x, count, tp, bundles, top, z, features, limbs, None)
    for wrong in (dict(limbs=3), dict(count=65537), dict(bundles=65537), dict(top=65537), dict(features=524281), dict(g=None),
                  dict(x=None), dict(tp=None), dict(z=None), dict(g=gates.data_ptr() + 4), dict(x=y.data_ptr() + 8),
                  dict(tp=terms.data_ptr() + 1), dict(z=to.data_ptr() + 4), dict(z=y.data_ptr()), dict(z=gates.data_ptr())):
        assert total(**wrong) == bad, wrong
        assert ck.ckks_last_error()
    with pytest.raises(ValueError):
        ck.ckks_experts_combine(ctx, gates, y[:2], terms, to, d_out, 2)
    with pytest.raises(ValueError):
        ck.ckks_experts_combine(ctx, gates, y, terms.to(torch.int64), to, d_out, 2)
    with pytest.raises(ValueError):
        ck.ckks_experts_combine(ctx, gates, y, terms, to[:1], d_out, 2)
