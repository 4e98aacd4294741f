"""GPU parity of the layer over 8-bit floating-point weights against the oracle,
bit for bit (residues have one right value, so there is no tolerance): every
code, ragged blocks, tiles and steps, one input and one output, the largest sums
that valid inputs give, offsets past 32 bits, and the refusals."""
import ctypes

import numpy as np
import pytest

from oracle import fp8 as OF
from workloads import gen

gpu = pytest.mark.gpu

_CTX = {}
MANY = 16   # limbs of 2^10 that make enough columns for the kernels of wide batches
CODES = np.array([c for c in range(256) if c & 0x7F != 0x7F], np.uint8)


def ctx_for(ck, log_n, limbs):
    key = (log_n, limbs)
    if key not in _CTX:
        _CTX[key] = ck.Context(log_n, limbs)
    return _CTX[key]


def layer(seed, d_out, d_in, block_rows=128):
    rng = np.random.default_rng(seed)
    codes = CODES[rng.integers(0, len(CODES), (d_out, d_in))]
    scales = rng.normal(0, 2e-4, (-(-d_out // block_rows), -(-d_in // OF.BLOCK))).astype(np.float32)
    return codes, scales


def encode(ck, ctx, codes, scales, block_rows, limbs, scale, bad=None):
    d_out, d_in = codes.shape
    enc = ck.empty_workspace(ck.ckks_fp8_weight_bytes(ctx, d_out, d_in, limbs))
    enc.fill_(-1)
    ck.ckks_linear_encode_fp8(ctx, ck.to_device(codes), ck.to_device(scales), d_out, d_in, block_rows, limbs, scale, enc, bad)
    return enc


def run(ck, ctx, codes, scales, ct, block_rows, scale):
    d_out, d_in = codes.shape
    limbs = ct.shape[2]
    enc = encode(ck, ctx, codes, scales, block_rows, limbs, scale)
    out = ck.empty_u32((d_out,) + tuple(ct.shape[1:]))
    out.fill_(-1)
    ck.ckks_linear_mac_fp8(ctx, enc, ct if hasattr(ct, "is_cuda") else ck.to_device(ct), out, d_out, d_in, limbs)
    return out


def check(ck, log_n, limbs, d_out, d_in, seed, block_rows=128, scale=2.0 ** 30, limbs_used=None, rows=None):
    ctx = ctx_for(ck, log_n, limbs)
    qs = ctx.moduli[:limbs_used or limbs]
    codes, scales = layer(seed, d_out, d_in, block_rows)
    ct = gen.uniform_residues(np.random.default_rng(seed + 1), (d_in, 2), qs, ctx.n)
    got = ck.to_host_u32(run(ck, ctx, codes, scales, ct, block_rows, scale))
    rows = list(range(d_out)) if rows is None else rows
    want = OF.mac(codes, scales, ct, block_rows, scale, qs, rows=rows).astype(np.uint32)
    assert np.array_equal(got[rows], want)
    assert np.all(got < np.array(qs, np.uint32)[None, None, :, None])


def check_many(ck, d_out, d_in, seed, block_rows=128):
    ctx = ctx_for(ck, 10, MANY)
    codes, scales = layer(seed, d_out, d_in, block_rows)
    ct = gen.uniform_residues(np.random.default_rng(seed + 1), (d_in, 2), ctx.moduli, ctx.n)
    got = ck.to_host_u32(run(ck, ctx, codes, scales, ct, block_rows, 2.0 ** 30))
    cols = [0, 31, 32, 63, 64, 500, 1023]
    rows = list(range(d_out)) if d_out <= 33 else [0, 31, 32, d_out // 2, d_out - 1]
    want = OF.mac(codes, scales, ct[..., cols], block_rows, 2.0 ** 30, ctx.moduli, rows=rows).astype(np.uint32)
    assert np.array_equal(got[rows][..., cols], want)
    assert np.all(got < np.array(ctx.moduli, np.uint32)[None, None, :, None])


@gpu
def test_every_code(gpu_lib):
    """One input, so that output j is code j's weight times it; NaN counts as zero."""
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    codes = np.arange(256, dtype=np.uint8).reshape(256, 1)
    ct = gen.uniform_residues(np.random.default_rng(1), (1, 2), ctx.moduli, ctx.n)
    scales = np.ones((2, 1), np.float32)
    got = ck.to_host_u32(run(ck, ctx, codes, scales, ct, 128, 64.0 * 12345))
    assert np.array_equal(got, OF.mac(codes, scales, ct, 128, 64.0 * 12345, ctx.moduli).astype(np.uint32))
    assert not got[0x7F].any() and not got[0xFF].any()


@gpu
@pytest.mark.parametrize("d_in", [1, 2, 15, 16, 17, 31, 32, 33, 63, 65, 96, 97, 127, 128, 129, 255, 257, 1023, 1024, 1025])
def test_input_counts(gpu_lib, d_in):
    check(gpu_lib, 10, 1, 18, d_in, 200 + d_in)


@gpu
@pytest.mark.parametrize("d_out", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 130, 257, 513, 600])
def test_output_counts(gpu_lib, d_out):
    check(gpu_lib, 10, 2, d_out, 70, 300 + d_out)


@gpu
@pytest.mark.parametrize("block_rows", [1, 7, 32, 64, 100, 128, 129, 4000])
@pytest.mark.parametrize("d_out,d_in", [(130, 300), (257, 128)])
def test_block_rows(gpu_lib, d_out, d_in, block_rows):
    check(gpu_lib, 10, 2, d_out, d_in, 350 + block_rows, block_rows)


@gpu
@pytest.mark.parametrize("d_in,d_out", [(1, 1), (16, 8), (17, 9), (31, 31), (64, 16), (300, 3), (700, 13), (1025, 1), (2500, 32),
                                        (300, 33), (64, 64), (129, 65)])
def test_few_outputs_of_many_columns(gpu_lib, d_in, d_out):
    check_many(gpu_lib, d_out, d_in, 460 + d_in)


@gpu
@pytest.mark.parametrize("d_in,d_out", [(1, 300), (40, 129), (65, 70), (320, 257), (500, 129), (512, 300), (513, 260), (640, 257),
                                        (1024, 290), (1025, 257), (1300, 513)])
def test_many_outputs_of_many_columns(gpu_lib, d_in, d_out):
    check_many(gpu_lib, d_out, d_in, 480 + d_in, 1 if d_in % 2 else 128)


@gpu
@pytest.mark.parametrize("d_in", [40, 250, 300, 512, 600, 1000, 1024, 1100, 1280])
@pytest.mark.parametrize("d_out", [290, 380, 420, 512, 530])
def test_row_tiles_and_passes(gpu_lib, d_out, d_in):
    """Whole passes over the row tiles, and rests of one to seven tiles that waves share or do not, with the
    inputs of one and of several chunks in LDS."""
    check_many(gpu_lib, d_out, d_in, 490 + d_in + d_out)


@gpu
@pytest.mark.parametrize("d_out,d_in", [(290, 40), (380, 40), (380, 250), (512, 250), (290, 512), (420, 512), (290, 1000), (380, 1000),
                                        (420, 1000), (530, 1024), (380, 1100), (290, 1280), (64, 300), (160, 1100)])
def test_every_row_tile_and_column_wave(gpu_lib, d_out, d_in):
    """The first and the last row of every row tile, at columns of each of the four waves that are next to each other: a tile or
    strip that was taken for another one gives residues in range, which only its own rows and columns show."""
    ck = gpu_lib
    ctx = ctx_for(ck, 10, MANY)
    codes, scales = layer(498 + d_in + d_out, d_out, d_in)
    ct = gen.uniform_residues(np.random.default_rng(499 + d_in), (d_in, 2), ctx.moduli, ctx.n)
    got = ck.to_host_u32(run(ck, ctx, codes, scales, ct, 128, 2.0 ** 30))
    rows = sorted({min(r, d_out - 1) for t in range(0, d_out, 32) for r in (t, t + 31)})
    cols = [3, 38, 75, 127, 130, 161, 192, 255, 515, 550, 580, 639, 897, 930, 975, 1020]
    of_rows = scales[np.array(rows) // 128]
    want = OF.mac(codes[rows], of_rows, ct[..., cols], 1, 2.0 ** 30, ctx.moduli).astype(np.uint32)
    assert np.array_equal(got[rows][..., cols], want)


@gpu
@pytest.mark.parametrize("log_n,limbs", [(10, 1), (10, 3), (11, 2), (12, 2)])
@pytest.mark.parametrize("d_out,d_in", [(9, 1500), (33, 700), (200, 130), (700, 300), (900, 900), (1100, 1100), (1500, 40)])
def test_few_columns(gpu_lib, log_n, limbs, d_out, d_in):
    """Inputs in shares that are summed, and rows split over workgroups."""
    check(gpu_lib, log_n, limbs, d_out, d_in, 495 + d_in, rows=sorted({0, 7, 31 % d_out, d_out // 2, d_out - 2, d_out - 1}))


@gpu
@pytest.mark.parametrize("d_in", [1152, 2048, 2049, 2500, 4100, 9000])
def test_deep_contractions(gpu_lib, d_in):
    check(gpu_lib, 10, 1, 70, d_in, 400 + d_in, rows=[0, 1, 16, 33, 69])


@gpu
@pytest.mark.parametrize("log_n,limbs", [(10, 1), (11, 3), (12, 16), (13, 4), (14, 2), (15, 2), (16, 2)])
def test_rings(gpu_lib, log_n, limbs):
    check(gpu_lib, log_n, limbs, 20, 40, 500 + log_n)


@gpu
def test_fewer_limbs_than_the_context(gpu_lib):
    check(gpu_lib, 11, 4, 33, 165, 520, limbs_used=2)


def largest_sums(ck, limbs, d_out, code, d_in):
    """Every weight at an end of its range (28672 units) or of its low digit's (1920 = 8 * 256 - 128), every
    input at an end of the digits' range or q - 1, and scales whose constants are the largest centred
    residues: 2^32, 2^48 or 2^64 times the first prime's are (q - 1) / 2 or (q + 1) / 2."""
    import torch
    ctx = ctx_for(ck, 10, limbs)
    codes = np.full((d_out, d_in), code, np.uint8)
    q = ctx.moduli[0]
    for residue in (0x3F7F7F7F, 0x3F7F7F80, None):
        ct = np.empty((d_in, 2, limbs, ctx.n), np.uint32)
        ct[:] = np.array(ctx.moduli, np.uint32)[:, None] - 1 if residue is None else residue
        assert residue is None or residue < min(ctx.moduli)
        d_ct = ck.to_device(ct)
        for shift in (32, 48, 64):
            for half in ((q - 1) // 2, (q + 1) // 2):
                s = half * pow(2, -shift, q) % q
                scales = np.ones((-(-d_out // 128), -(-d_in // 128)), np.float32)
                got = run(ck, ctx, codes, scales, d_ct, 128, 64.0 * s)
                want = OF.mac(codes[:1], scales[:1], ct[..., :1], 128, 64.0 * s, ctx.moduli).astype(np.int32)
                assert bool((got == torch.from_numpy(want).cuda()).all()), (residue, shift, half)


@gpu
@pytest.mark.parametrize("d_in", [128, 1024, 1100, 2100])
@pytest.mark.parametrize("code", [0x7E, 0xFE, 0x5F, 0xDF])
@pytest.mark.parametrize("limbs,d_out", [(1, 4), (1, 300), (MANY, 4), (MANY, 300)])
def test_the_largest_sums(gpu_lib, limbs, d_out, code, d_in):
    largest_sums(gpu_lib, limbs, d_out, code, d_in)


@gpu
@pytest.mark.parametrize("d_in", [256, 384, 512])
@pytest.mark.parametrize("code", [0x7E, 0xFE, 0x5F, 0xDF])
def test_the_largest_sums_of_few_blocks(gpu_lib, code, d_in):
    largest_sums(gpu_lib, MANY, 300, code, d_in)


@gpu
def test_huge_scales(gpu_lib):
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    codes, _ = layer(525, 9, 300)
    scales = np.array([[1.75 * 2.0 ** 62, -(2.0 ** 62), 3.0]], np.float32)
    ct = gen.uniform_residues(np.random.default_rng(526), (300, 2), ctx.moduli, ctx.n)
    got = ck.to_host_u32(run(ck, ctx, codes, scales, ct, 128, 64.0))
    assert np.array_equal(got, OF.mac(codes, scales, ct, 128, 64.0, ctx.moduli).astype(np.uint32))


@gpu
def test_scales_past_63_bits_are_counted(gpu_lib):
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    codes, _ = layer(527, 9, 640)
    scales = np.array([[2.0 ** 63, -(2.0 ** 63), np.nextafter(np.float32(2.0 ** 63), np.float32(0)), 3e38, 3.0]], np.float32)
    bad = torch.zeros(1, dtype=torch.int32, device="cuda")
    enc = encode(ck, ctx, codes, scales, 128, 2, 64.0, bad)
    assert int(bad) == 3
    ct = gen.uniform_residues(np.random.default_rng(528), (640, 2), ctx.moduli, ctx.n)
    out = ck.empty_u32((9, 2, 2, ctx.n))
    ck.ckks_linear_mac_fp8(ctx, enc, ck.to_device(ct), out, 9, 640, 2)
    assert np.array_equal(ck.to_host_u32(out), OF.mac(codes, scales, ct, 128, 64.0, ctx.moduli).astype(np.uint32))


@gpu
def test_scales_that_round_to_zero_are_counted(gpu_lib):
    """Halves go to zero (to even); zeros are what they are."""
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    codes, _ = layer(533, 70, 700)
    scales = np.array([[0.0, -0.0, 0.5, -0.25, 1e-42, 0.51], [1.0, -0.5, 0.5000001, 0.0, -1e-30, 3.0], [2.0] * 6], np.float32)
    bad = torch.zeros(1, dtype=torch.int32, device="cuda")
    enc = encode(ck, ctx, codes, scales, 32, 2, 64.0, bad)
    assert int(bad) == 5
    ct = gen.uniform_residues(np.random.default_rng(534), (700, 2), ctx.moduli, ctx.n)
    out = ck.empty_u32((70, 2, 2, ctx.n))
    ck.ckks_linear_mac_fp8(ctx, enc, ck.to_device(ct), out, 70, 700, 2)
    assert np.array_equal(ck.to_host_u32(out), OF.mac(codes, scales, ct, 32, 64.0, ctx.moduli).astype(np.uint32))


@gpu
def test_what_is_no_number_is_counted(gpu_lib):
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    codes, scales = layer(530, 300, 200, 64)
    codes[0, 0] = codes[299, 199] = codes[64, 128] = 0x7F
    codes[100, 5] = 0xFF
    scales[0, 1], scales[4, 0], scales[2, 0] = np.inf, np.nan, -np.inf
    bad = torch.full((1,), 77, dtype=torch.int32, device="cuda")
    for _ in range(2):
        enc = encode(ck, ctx, codes, scales, 64, 2, 2.0 ** 30, bad)
        assert int(bad) == 7
    ct = gen.uniform_residues(np.random.default_rng(531), (200, 2), ctx.moduli, ctx.n)
    out = ck.empty_u32((300, 2, 2, ctx.n))
    ck.ckks_linear_mac_fp8(ctx, enc, ck.to_device(ct), out, 300, 200, 2)
    assert np.array_equal(ck.to_host_u32(out), OF.mac(codes, scales, ct, 64, 2.0 ** 30, ctx.moduli).astype(np.uint32))
    ok_codes, ok_scales = layer(532, 3, 40)
    encode(ck, ctx, ok_codes, ok_scales, 128, 2, 2.0 ** 30, bad)
    assert int(bad) == 0


@gpu
@pytest.mark.parametrize("d_out,d_in", [(70, 1100), (600, 1030), (6, 1100), (1200, 30)])
def test_offsets_past_32_bits(gpu_lib, d_out, d_in):
    """Rows of 4 MiB: the inputs (and the outputs) pass 2^32 bytes; checked on a sample of columns."""
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 16, 8)
    codes, scales = layer(540, d_out, d_in)
    g = torch.Generator(device="cuda").manual_seed(5)
    ct = torch.empty((d_in, 2, 8, ctx.n), dtype=torch.int32, device="cuda")
    for l, q in enumerate(ctx.moduli):
        ct[:, :, l] = torch.randint(0, q, (d_in, 2, ctx.n), generator=g, device="cuda", dtype=torch.int32)
    out = run(ck, ctx, codes, scales, ct, 128, 2.0 ** 31)
    cols = torch.tensor([0, 1, 4097, 32768, 65535], device="cuda")
    rows = sorted({0, 1, 5, d_out // 2, d_out - 2, d_out - 1})
    got = out[rows][..., cols].cpu().numpy().view(np.uint32)
    part = ct[..., cols].cpu().numpy().view(np.uint32)
    assert np.array_equal(got, OF.mac(codes, scales, part, 128, 2.0 ** 31, ctx.moduli, rows=rows).astype(np.uint32))


@gpu
def test_unaligned_weights_another_stream_and_a_graph(gpu_lib):
    """Weights at an odd address, as float8_e4m3fn; the calls on a stream of their own; a graph of both, replayed
    with eager work between, equals the eager result every time."""
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 11, 2)
    d_out, d_in = 66, 129
    codes, scales = layer(550, d_out, d_in, 64)
    ct = gen.uniform_residues(np.random.default_rng(551), (d_in, 2), ctx.moduli, ctx.n)
    want = OF.mac(codes, scales, ct, 64, 2.0 ** 30, ctx.moduli).astype(np.uint32)
    w8 = torch.empty(codes.size + 1, dtype=torch.uint8, device="cuda")[1:].view(codes.shape)
    w8.copy_(torch.from_numpy(codes))
    w8 = w8.view(torch.float8_e4m3fn)
    d_s, d_ct = ck.to_device(scales), ck.to_device(ct)
    enc = ck.empty_workspace(ck.ckks_fp8_weight_bytes(ctx, d_out, d_in, 2))
    bad = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = ck.empty_u32((d_out, 2, 2, ctx.n))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def calls():
        ck.ckks_linear_encode_fp8(ctx, w8, d_s, d_out, d_in, 64, 2, 2.0 ** 30, enc, bad, stream=s)
        ck.ckks_linear_mac_fp8(ctx, enc, d_ct, out, d_out, d_in, 2, stream=s)
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
        bad.fill_(9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(ck.to_host_u32(out), want) and int(bad) == 0
        ck.ckks_linear_mac_fp8(ctx, enc, d_ct, other, d_out, d_in, 2)
        torch.cuda.synchronize()
    assert np.array_equal(ck.to_host_u32(other), want)
    del graph


@gpu
def test_empty_layers(gpu_lib):
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    out = ck.empty_u32((3, 2, 2, ctx.n))
    out.fill_(-1)
    ck.ckks_linear_mac_fp8(ctx, None, None, out, 3, 0, 2)
    assert np.all(ck.to_host_u32(out) == 0)
    assert ck.ckks_fp8_weight_bytes(ctx, 3, 0, 2) == 0 and ck.ckks_fp8_weight_bytes(ctx, 0, 3, 2) == 0
    out.fill_(7)
    ck.ckks_linear_mac_fp8(ctx, None, None, out, 0, 5, 2)
    bad = torch.full((1,), 5, dtype=torch.int32, device="cuda")
    ck.ckks_linear_encode_fp8(ctx, None, None, 0, 5, 128, 2, 1.0, None, bad)
    assert np.all(ck.to_host_u32(out) == 7) and int(bad) == 0


@gpu
@pytest.mark.parametrize("limbs", [1, 2])
def test_weight_bytes_are_as_declared(gpu_lib, limbs):
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    for d_out, d_in in [(1, 1), (32, 32), (33, 128), (100, 129), (513, 1021), (768, 2048)]:
        rows, inputs = -(-d_out // 32) * 32, -(-d_in // 32) * 32
        assert ck.ckks_fp8_weight_bytes(ctx, d_out, d_in, limbs) == 2 * rows * inputs + 12 * limbs * rows * -(-d_in // 128)


@gpu
def test_refusals(gpu_lib):
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    d_out, d_in = 16, 64
    codes, scales = layer(560, d_out, d_in)
    w8, d_s = ck.to_device(codes), ck.to_device(scales)
    enc = ck.empty_workspace(ck.ckks_fp8_weight_bytes(ctx, d_out, d_in, 2))
    ct, out = ck.empty_u32((d_in, 2, 2, ctx.n)), ck.empty_u32((d_out, 2, 2, ctx.n))
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(ck.CkksError) as e:
            ck.ckks_linear_encode_fp8(ctx, w8, d_s, d_out, d_in, 128, 2, scale, enc)
        assert e.value.code == ck.CKKS_E_INVALID_ARG
    raw, bad = ck._lib.ckks_linear_encode_fp8, ck.CKKS_E_INVALID_ARG
    at = (w8.data_ptr(), d_s.data_ptr())
    assert raw(ctx.handle, *at, d_out, d_in, 0, 2, 1.0, enc.data_ptr(), None, None) == bad
    assert raw(ctx.handle, *at, d_out, d_in, 128, 3, 1.0, enc.data_ptr(), None, None) == bad
    assert raw(ctx.handle, None, at[1], d_out, d_in, 128, 2, 1.0, enc.data_ptr(), None, None) == bad
    assert raw(ctx.handle, at[0], at[1] + 2, d_out, d_in, 128, 2, 1.0, enc.data_ptr(), None, None) == bad
    assert raw(ctx.handle, *at, d_out, d_in, 128, 2, 1.0, enc.data_ptr() + 8, None, None) == bad
    assert raw(ctx.handle, *at, d_out, d_in, 128, 2, 1.0, enc.data_ptr(), enc.data_ptr() + 4, None) == bad
    assert "overlaps" in ck.ckks_last_error()
    assert raw(ctx.handle, enc.data_ptr(), at[1], d_out, d_in, 128, 2, 1.0, enc.data_ptr(), None, None) == bad
    raw = ck._lib.ckks_linear_mac_fp8
    at = (enc.data_ptr(), ct.data_ptr(), out.data_ptr())
    assert raw(ctx.handle, *at, d_out, d_in, 3, None) == bad            # limbs
    assert raw(ctx.handle, *at, 524281, d_in, 2, None) == bad
    assert raw(ctx.handle, *at, d_out, (1 << 24) + 1, 2, None) == bad
    assert raw(ctx.handle, None, at[1], at[2], d_out, d_in, 2, None) == bad
    assert raw(ctx.handle, at[0] + 4, at[1], at[2], d_out, d_in, 2, None) == bad
    assert raw(ctx.handle, at[0], at[1], at[1], d_out, d_in, 2, None) == bad
    assert "overlaps" in ck.ckks_last_error()
    assert raw(ctx.handle, at[0], at[1], at[0], d_out, d_in, 2, None) == bad
    with pytest.raises(ValueError):   # half the inputs
        ck.ckks_linear_mac_fp8(ctx, enc, ct[:32], out, d_out, d_in, 2)
    with pytest.raises(ValueError):   # encoded for fewer outputs
        ck.ckks_linear_mac_fp8(ctx, enc[:4], ct, out, d_out, d_in, 2)
    for other in (w8.view(torch.int8), w8.view(torch.float8_e5m2), w8.view(torch.float8_e4m3fnuz)):
        with pytest.raises(ValueError):
            ck.ckks_linear_encode_fp8(ctx, other, d_s, d_out, d_in, 128, 2, 1.0, enc)
    with pytest.raises(ValueError):   # scales of whole numbers
        ck.ckks_linear_encode_fp8(ctx, w8, d_s.view(torch.int32), d_out, d_in, 128, 2, 1.0, enc)
    with pytest.raises(ValueError):
        ck.ckks_linear_encode_fp8(ctx, w8[:, ::2], d_s, d_out, d_in // 2, 128, 2, 1.0, enc)
    with pytest.raises(ValueError):   # a scale a row, and there is one
        ck.ckks_linear_encode_fp8(ctx, w8, d_s, d_out, d_in, 1, 2, 1.0, enc)
    with pytest.raises(ValueError):
        ck.ckks_fp8_weight_bytes(ctx, d_out, d_in, 3)


@gpu
def test_counts_of_other_types_are_refused(gpu_lib):
    """Four bytes wide, but no int32: a float would hold the count's bits, not the count."""
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 1)
    codes, scales = layer(565, 8, 32)
    with pytest.raises(ValueError, match="bad must be int32"):
        encode(ck, ctx, codes, scales, 128, 1, 2.0 ** 30, torch.zeros(1, device="cuda"))
    enc = encode(ck, ctx, codes, scales, 128, 1, 2.0 ** 30).view(1, -1)
    ct, out = ck.empty_u32((1, 32, 2, 1, ctx.n)), ck.empty_u32((1, 8, 2, 1, ctx.n))
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="status must be int32"):
        ck.ckks_experts_mac_fp8(ctx, enc, one, one, ct, out, 8, 32, 1, torch.zeros(1, device="cuda"))


def test_null_context_is_rejected_without_a_gpu():
    import paper_2606_17421_amd as ck
    lib, bad = ck._lib, ck.CKKS_E_INVALID_ARG
    assert lib.ckks_linear_mac_fp8(None, None, None, None, 1, 1, 1, None) == bad
    assert lib.ckks_linear_encode_fp8(None, None, None, 1, 1, 128, 1, 1.0, None, None, None) == bad
    assert lib.ckks_fp8_weight_bytes(None, 1, 1, 1) == ctypes.c_size_t(-1).value
    assert lib.ckks_experts_mac_fp8(None, None, 1, None, None, 1, None, 1, None, 1, 1, 1, None, None) == bad
    assert lib.ckks_experts_combine(None, None, None, 1, None, 1, 1, None, 1, 1, None) == bad
