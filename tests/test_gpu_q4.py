"""GPU parity of the layer over 4-bit weights against the oracle, bit for bit
(residues have one right value, so there is no tolerance): every group kind,
ragged groups, tiles and steps, one input and one output, zero points, the
largest sums that valid inputs give, offsets past 32 bits, and the refusals."""
import numpy as np
import pytest

from oracle import q4 as OQ
from workloads import gen

gpu = pytest.mark.gpu

_CTX = {}


def ctx_for(ck, log_n, limbs):
    key = (log_n, limbs)
    if key not in _CTX:
        _CTX[key] = ck.Context(log_n, limbs)
    return _CTX[key]


def layer(seed, d_out, d_in, group, zeros):
    rng = np.random.default_rng(seed)
    groups = -(-d_in // group)
    u = rng.integers(0, 16, (d_out, d_in))
    scales = (rng.normal(0, 0.01, (d_out, groups))).astype(np.float32)
    z = rng.integers(0, 16, (d_out, groups)).astype(np.uint8) if zeros else None
    return OQ.pack(u), scales, z


def encode(ck, ctx, w4, scales, z, d_out, d_in, group, limbs, scale):
    need = ck.ckks_q4_weight_bytes(ctx, d_out, d_in, group, limbs, z is not None)
    enc = ck.empty_workspace(need)
    enc.fill_(-1)
    ck.ckks_linear_encode_q4(ctx, ck.to_device(w4), ck.to_device(scales), None if z is None else ck.to_device(z), d_out,
                             d_in, group, limbs, scale, enc)
    return enc


def run(ck, ctx, w4, scales, z, ct, d_out, group, scale):
    d_in, _, limbs, n = ct.shape
    enc = encode(ck, ctx, w4, scales, z, d_out, d_in, group, limbs, scale)
    out = ck.empty_u32((d_out, 2, limbs, n))
    out.fill_(-1)
    ck.ckks_linear_mac_q4(ctx, enc, ck.to_device(ct), out, d_out, d_in, group, limbs, z is not None)
    return ck.to_host_u32(out)


def check(ck, log_n, limbs, d_out, d_in, group, zeros, seed, scale=2.0 ** 26, limbs_used=None, rows=None):
    ctx = ctx_for(ck, log_n, limbs)
    used = limbs_used or limbs
    qs = ctx.moduli[:used]
    w4, scales, z = layer(seed, d_out, d_in, group, zeros)
    ct = gen.uniform_residues(np.random.default_rng(seed + 1), (d_in, 2), qs, ctx.n)
    got = run(ck, ctx, w4, scales, z, ct, d_out, group, scale)
    rows = list(range(d_out)) if rows is None else rows
    want = OQ.mac(w4, scales, z, ct, group, scale, qs, rows=rows).astype(np.uint32)
    assert np.array_equal(got[rows], want)
    assert np.all(got < np.array(qs, np.uint32)[None, None, :, None])


@gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 96, 128, 192, 256, 320, 512, 1024])
def test_groups(gpu_lib, group, zeros):
    check(gpu_lib, 10, 2, 37, 1100, group, zeros, 100 + group)


@gpu
@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("d_in", [1, 2, 31, 32, 33, 63, 65, 127, 129, 255, 257, 1023, 1024, 1025])
def test_input_counts(gpu_lib, d_in, group):
    check(gpu_lib, 10, 1, 18, d_in, group, (d_in + group) % 3 == 0, 200 + d_in)


@gpu
@pytest.mark.parametrize("d_out", [1, 15, 16, 17, 63, 64, 65, 128, 130, 257, 513, 600])
def test_output_counts(gpu_lib, d_out):
    check(gpu_lib, 10, 2, d_out, 70, 64, d_out % 2 == 1, 300 + d_out)


@gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("d_in,group", [(70, 128), (96, 96), (513, 96), (1000, 192), (1024, 96), (1025, 96), (2500, 288)])
def test_groups_of_three_steps(gpu_lib, d_in, group, zeros):
    """Groups of 96 inputs and their multiples in a strip that stays whole (1024 inputs end inside
    the last group, a step past them) and in chunks."""
    check(gpu_lib, 10, 1, 300, d_in, group, zeros, 450 + d_in, rows=[0, 31, 64, 255, 299])


MANY = 16   # limbs of 2^10 that make enough columns for the kernels of wide batches


def check_many(ck, d_out, d_in, group, zeros, seed):
    ctx = ctx_for(ck, 10, MANY)
    w4, scales, z = layer(seed, d_out, d_in, group, zeros)
    ct = gen.uniform_residues(np.random.default_rng(seed + 1), (d_in, 2), ctx.moduli, ctx.n)
    got = run(ck, ctx, w4, scales, z, ct, d_out, group, 2.0 ** 26)
    cols = [0, 31, 32, 63, 64, 500, 1023]
    rows = list(range(d_out)) if d_out <= 32 else [0, 31, 32, d_out // 2, d_out - 1]
    want = OQ.mac(w4, scales, z, ct[..., cols], group, 2.0 ** 26, ctx.moduli, rows=rows).astype(np.uint32)
    assert np.array_equal(got[rows][..., cols], want)
    assert np.all(got < np.array(ctx.moduli, np.uint32)[None, None, :, None])


@gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 96, 128])
@pytest.mark.parametrize("d_in,d_out", [(1, 1), (16, 8), (17, 9), (31, 31), (64, 16), (300, 3), (700, 13), (1025, 1), (2500, 16)])
def test_few_outputs_of_many_columns(gpu_lib, d_in, d_out, group, zeros):
    check_many(gpu_lib, d_out, d_in, group, zeros, 460 + d_in)


@gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 96, 128])
@pytest.mark.parametrize("d_in,d_out", [(1, 33), (40, 64), (33, 31), (65, 9), (320, 70), (321, 128), (200, 300), (500, 129), (640, 257), (641, 200)])
def test_short_inputs_of_many_columns(gpu_lib, d_in, d_out, group, zeros):
    check_many(gpu_lib, d_out, d_in, group, zeros, 480 + d_in)


@gpu
@pytest.mark.parametrize("d_in,group", [(2048, 128), (2049, 64), (3072, 256), (4100, 32), (9000, 128), (2100, 2112)])
@pytest.mark.parametrize("zeros", [False, True])
def test_deep_contractions(gpu_lib, d_in, group, zeros):
    check(gpu_lib, 10, 1, 70, d_in, group, zeros, 400 + d_in, rows=[0, 1, 16, 33, 69])


@gpu
@pytest.mark.parametrize("log_n,limbs", [(10, 1), (11, 3), (12, 16), (13, 4), (14, 2), (15, 2), (16, 2)])
def test_rings(gpu_lib, log_n, limbs):
    check(gpu_lib, log_n, limbs, 20, 40, 32, log_n % 2 == 0, 500 + log_n)


@gpu
def test_fewer_limbs_than_the_context(gpu_lib):
    check(gpu_lib, 11, 4, 33, 65, 64, False, 520, limbs_used=2)


@gpu
@pytest.mark.parametrize("group,d_in", [(32, 1024), (64, 1024), (128, 2048), (256, 1024), (256, 1300), (1024, 1024)])
@pytest.mark.parametrize("residue", [0x3F7F7F7F, 0x3F7F7F80, None])
@pytest.mark.parametrize("u,z", [(0, None), (15, None), (0, 15), (15, 0)])
@pytest.mark.parametrize("limbs", [1, MANY])
def test_the_largest_sums(gpu_lib, u, z, residue, group, d_in, limbs):
    """Every input at an end of the digits' range (None: q - 1), every weight at an end of its, and a
    scale of +-8 units, whose sixteenth is the largest centred residue; and scales of 2^61."""
    ck = gpu_lib
    ctx = ctx_for(ck, 10, limbs)
    groups = -(-d_in // group)
    top = np.array(ctx.moduli, np.uint32)[None, None, :, None] - 1
    ct = np.broadcast_to(top if residue is None else np.uint32(residue), (d_in, 2, limbs, ctx.n)).copy()
    assert np.all(ct <= top)
    scales = np.empty((4, groups), np.float32)
    scales[0], scales[1], scales[2], scales[3] = 8, -8, 1.75 * 2.0 ** 61, -(2.0 ** 62)
    w4 = OQ.pack(np.full((4, d_in), u))
    zz = None if z is None else np.full((4, groups), z, np.uint8)
    got = run(ck, ctx, w4, scales, zz, ct, 4, group, 1.0)
    want = OQ.mac(w4, scales, zz, ct[..., :1], group, 1.0, ctx.moduli).astype(np.uint32)
    assert np.array_equal(got, np.broadcast_to(want, got.shape))


@gpu
def test_zero_points_count_four_bits(gpu_lib):
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 1)
    w4, scales, z = layer(530, 16, 64, 32, True)
    ct = gen.uniform_residues(np.random.default_rng(531), (64, 2), ctx.moduli, ctx.n)
    a = run(ck, ctx, w4, scales, z, ct, 16, 32, 2.0 ** 26)
    b = run(ck, ctx, w4, scales, z | 0xA0, ct, 16, 32, 2.0 ** 26)
    assert np.array_equal(a, b)


@gpu
@pytest.mark.parametrize("d_out,d_in,group,zeros", [(70, 1100, 128, False), (600, 1030, 64, True), (6, 1100, 96, True), (1200, 30, 32, False)])
def test_offsets_past_32_bits(gpu_lib, d_out, d_in, group, zeros):
    """Rows of 4 MiB: the inputs (and the outputs) pass 2^32 bytes; checked on a sample of columns."""
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 16, 8)
    w4, scales, z = layer(540, d_out, d_in, group, zeros)
    g = torch.Generator(device="cuda").manual_seed(5)
    ct = torch.empty((d_in, 2, 8, ctx.n), dtype=torch.int32, device="cuda")
    for l, q in enumerate(ctx.moduli):
        ct[:, :, l] = torch.randint(0, q, (d_in, 2, ctx.n), generator=g, device="cuda", dtype=torch.int32)
    enc = encode(ck, ctx, w4, scales, z, d_out, d_in, group, 8, 2.0 ** 28)
    out = ck.empty_u32((d_out, 2, 8, ctx.n))
    ck.ckks_linear_mac_q4(ctx, enc, ct, out, d_out, d_in, group, 8, zeros)
    cols = torch.tensor([0, 1, 4097, 32768, 65535], device="cuda")
    got = out[..., cols].cpu().numpy().view(np.uint32)
    part = ct[..., cols].cpu().numpy().view(np.uint32)
    want = OQ.mac(w4, scales, z, part, group, 2.0 ** 28, ctx.moduli).astype(np.uint32)
    assert np.array_equal(got, want)


@gpu
def test_unaligned_weights_another_stream_and_a_graph(gpu_lib):
    """4-bit weights and zero points at odd addresses; the calls on a stream of their own; a graph
    of both, replayed with eager work between, equals the eager result every time."""
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 11, 2)
    d_out, d_in, group = 66, 129, 64
    w4, scales, z = layer(550, d_out, d_in, group, True)
    ct = gen.uniform_residues(np.random.default_rng(551), (d_in, 2), ctx.moduli, ctx.n)
    want = OQ.mac(w4, scales, z, ct, group, 2.0 ** 26, ctx.moduli).astype(np.uint32)

    def odd(a):
        t = torch.empty(a.size + 1, dtype=torch.uint8, device="cuda")[1:].view(a.shape)
        t.copy_(torch.from_numpy(a))
        return t
    d_w4, d_z, d_s, d_ct = odd(w4), odd(z), ck.to_device(scales), ck.to_device(ct)
    enc = ck.empty_workspace(ck.ckks_q4_weight_bytes(ctx, d_out, d_in, group, 2, True))
    out = ck.empty_u32((d_out, 2, 2, ctx.n))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def calls():
        ck.ckks_linear_encode_q4(ctx, d_w4, d_s, d_z, d_out, d_in, group, 2, 2.0 ** 26, enc, stream=s)
        ck.ckks_linear_mac_q4(ctx, enc, d_ct, out, d_out, d_in, group, 2, True, stream=s)
    with torch.cuda.stream(s):
        calls()
    s.synchronize()
    assert np.array_equal(ck.to_host_u32(out), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        calls()
    other = ck.empty_u32((d_out, 2, 2, ctx.n))
    for _ in range(3):
        out.fill_(0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(ck.to_host_u32(out), want)
        ck.ckks_linear_mac_q4(ctx, enc, d_ct, other, d_out, d_in, group, 2, True)
        torch.cuda.synchronize()
    assert np.array_equal(ck.to_host_u32(other), want)
    del graph


@gpu
def test_empty_layers(gpu_lib):
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    out = ck.empty_u32((3, 2, 2, ctx.n))
    out.fill_(-1)
    ck.ckks_linear_mac_q4(ctx, None, None, out, 3, 0, 32, 2)
    assert np.all(ck.to_host_u32(out) == 0)
    assert ck.ckks_q4_weight_bytes(ctx, 3, 0, 32, 2) == 0
    out.fill_(7)
    ck.ckks_linear_mac_q4(ctx, None, None, out, 0, 5, 32, 2)
    ck.ckks_linear_encode_q4(ctx, None, None, None, 0, 5, 32, 2, 1.0, None)
    assert np.all(ck.to_host_u32(out) == 7)


@gpu
def test_refusals(gpu_lib):
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    d_out, d_in = 16, 64
    w4, scales, _ = layer(560, d_out, d_in, 32, False)
    d_w4, d_s = ck.to_device(w4), ck.to_device(scales)
    enc = ck.empty_workspace(ck.ckks_q4_weight_bytes(ctx, d_out, d_in, 32, 2))
    ct, out = ck.empty_u32((d_in, 2, 2, ctx.n)), ck.empty_u32((d_out, 2, 2, ctx.n))
    for group in (0, 1, 33, 48):
        with pytest.raises(ValueError):
            ck.ckks_q4_weight_bytes(ctx, d_out, d_in, group, 2)
        assert ck._lib.ckks_linear_mac_q4(ctx.handle, enc.data_ptr(), ct.data_ptr(), out.data_ptr(), d_out, d_in, group, 2,
                                          0, None) == ck.CKKS_E_INVALID_ARG
        assert "group" in ck.ckks_last_error()
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(ck.CkksError) as e:
            ck.ckks_linear_encode_q4(ctx, d_w4, d_s, None, d_out, d_in, 32, 2, scale, enc)
        assert e.value.code == ck.CKKS_E_INVALID_ARG
    raw = ck._lib.ckks_linear_mac_q4
    at = (enc.data_ptr(), ct.data_ptr(), out.data_ptr())
    assert raw(ctx.handle, *at, d_out, d_in, 32, 2, 2, None) == ck.CKKS_E_INVALID_ARG       # zeros is 0 or 1
    assert raw(ctx.handle, *at, d_out, d_in, 32, 3, 0, None) == ck.CKKS_E_INVALID_ARG       # limbs
    assert raw(ctx.handle, *at, 524281, d_in, 32, 2, 0, None) == ck.CKKS_E_INVALID_ARG
    assert raw(ctx.handle, *at, d_out, (1 << 24) + 1, 32, 2, 0, None) == ck.CKKS_E_INVALID_ARG
    assert raw(ctx.handle, None, at[1], at[2], d_out, d_in, 32, 2, 0, None) == ck.CKKS_E_INVALID_ARG
    assert raw(ctx.handle, at[0] + 4, at[1], at[2], d_out, d_in, 32, 2, 0, None) == ck.CKKS_E_INVALID_ARG
    assert raw(ctx.handle, at[0], at[1], at[1], d_out, d_in, 32, 2, 0, None) == ck.CKKS_E_INVALID_ARG
    assert "overlaps" in ck.ckks_last_error()
    assert raw(ctx.handle, at[0], at[1], at[0], d_out, d_in, 32, 2, 0, None) == ck.CKKS_E_INVALID_ARG
    with pytest.raises(ValueError):   # half the inputs
        ck.ckks_linear_mac_q4(ctx, enc, ct[:32], out, d_out, d_in, 32, 2)
    with pytest.raises(ValueError):   # encoded for fewer outputs
        ck.ckks_linear_mac_q4(ctx, enc[:4], ct, out, d_out, d_in, 32, 2)
    with pytest.raises(ValueError):   # scales of whole numbers
        ck.ckks_linear_encode_q4(ctx, d_w4, d_s.view(torch.int32), None, d_out, d_in, 32, 2, 1.0, enc)
    with pytest.raises(ValueError):
        ck.ckks_linear_encode_q4(ctx, d_w4[:, ::2], d_s, None, d_out, d_in // 2, 32, 2, 1.0, enc)
    whole = torch.empty(4096, dtype=torch.uint8, device="cuda")
    assert ck._lib.ckks_linear_encode_q4(ctx.handle, whole.data_ptr(), d_s.data_ptr(), None, d_out, d_in, 32, 2, 1.0,
                                         whole.data_ptr(), None) == ck.CKKS_E_INVALID_ARG


def test_null_context_is_rejected_without_a_gpu():
    import ctypes

    import paper_2606_17421_amd as ck
    lib = ck._lib
    assert lib.ckks_linear_mac_q4(None, None, None, None, 1, 1, 32, 1, 0, None) == ck.CKKS_E_INVALID_ARG
    assert lib.ckks_linear_encode_q4(None, None, None, None, 1, 1, 32, 1, 1.0, None, None) == ck.CKKS_E_INVALID_ARG
    assert lib.ckks_q4_weight_bytes(None, 1, 1, 32, 1, 0) == ctypes.c_size_t(-1).value


@gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("d_in,group", [(64, 0xFFFFFFE0), (33, 0xFFFFFFE0), (200, 0xFFFFFF80), (1100, 0xFFFFFFE0), (70, 1 << 31)])
def test_groups_far_longer_than_the_layer(gpu_lib, d_in, group, zeros):
    """A group that ends past 2^32 inputs is one scale and zero point a row, as one of the layer's length is."""
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    for kind in (False, True):
        assert ck.ckks_q4_weight_bytes(ctx, 5, d_in, group, 2, kind) == \
            ck.ckks_q4_weight_bytes(ctx, 5, d_in, -(-d_in // 32) * 32, 2, kind)
    check(ck, 10, 2, 5, d_in, group, zeros, 570 + d_in)


@gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("limbs", [1, 2])
def test_weight_bytes_are_as_declared(gpu_lib, limbs, zeros):
    """The header's formula: padded rows times padded inputs, and a pair of scales a row and s inputs."""
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    assert ck.ckks_q4_weight_bytes(ctx, 1, 128, 128, 2) == 5120
    for d_out, d_in, group, s in [(1, 128, 128, 128), (64, 768, 128, 128), (65, 769, 96, 96), (100, 200, 192, 96), (7, 300, 320, 128),
                                  (7, 33, 320, 64), (7, 70, 320, 96), (7, 5, 32, 32), (513, 1021, 32, 32), (3, 500, 320, 64),
                                  (3, 900, 160, 32)]:
        rows, inputs = -(-d_out // 64) * 64, -(-d_in // s) * s
        want = rows * inputs // (1 if zeros else 2) + 8 * limbs * rows * (inputs // s)
        assert ck.ckks_q4_weight_bytes(ctx, d_out, d_in, group, limbs, zeros) == want, (d_out, d_in, group)


@gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 96, 128])
@pytest.mark.parametrize("d_out", [7, 16])
def test_few_outputs_of_deep_layers_in_one_slice(gpu_lib, d_out, group, zeros):
    """Columns enough that one wave goes through all inputs, so that it reduces its sums twice on the
    way: random layers and the largest sums, checked on a sample of columns."""
    import torch
    ck = gpu_lib
    limbs, d_in = 8, 2100
    ctx = ctx_for(ck, 14, limbs)
    w4, scales, z = layer(580 + group, d_out, d_in, group, zeros)
    g = torch.Generator(device="cuda").manual_seed(group)
    ct = torch.empty((d_in, 2, limbs, ctx.n), dtype=torch.int32, device="cuda")
    for l, q in enumerate(ctx.moduli):
        ct[:, :, l] = torch.randint(0, q, (d_in, 2, ctx.n), generator=g, device="cuda", dtype=torch.int32)
    out = ck.empty_u32((d_out, 2, limbs, ctx.n))
    cols = torch.tensor([0, 1, 63, 64, 9000, 16383], device="cuda")

    def compare(w4, scales, z, scale):
        enc = encode(ck, ctx, w4, scales, z, d_out, d_in, group, limbs, scale)
        out.fill_(-1)
        ck.ckks_linear_mac_q4(ctx, enc, ct, out, d_out, d_in, group, limbs, zeros)
        got = out[..., cols].cpu().numpy().view(np.uint32)
        part = ct[..., cols].cpu().numpy().view(np.uint32)
        assert np.array_equal(got, OQ.mac(w4, scales, z, part, group, scale, ctx.moduli).astype(np.uint32))
    compare(w4, scales, z, 2.0 ** 26)
    ends = np.full_like(scales, 8)
    ends[1::2] = -8
    for residue in (0x3F7F7F7F, 0x3F7F7F80):
        assert residue < min(ctx.moduli)
        ct.fill_(residue)
        for u in (0, 15):
            compare(OQ.pack(np.full((d_out, d_in), u)), ends, np.full_like(z, 15 - u) if zeros else None, 1.0)
