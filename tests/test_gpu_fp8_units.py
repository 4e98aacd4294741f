"""GPU parity of the 8-bit layers' encode with a unit for each output and 128 inputs against the oracle, bit for bit,
in every kernel of the products: outputs of unlike sizes, ragged blocks, NaN, scales too small or too large, and the refusals."""
import numpy as np
import pytest

from oracle import fp8 as OF
from test_gpu_fp8 import MANY, ctx_for, encode as encode_64ths, layer
from workloads import gen

gpu = pytest.mark.gpu


def spread_layer(seed, d_out, d_in, block_rows=128):
    """Every row and block with a largest size of its own: at and one code past 56, 112 and 224, the largest, one of all sizes."""
    rng = np.random.default_rng(seed)
    codes, scales = layer(seed, d_out, d_in, block_rows)
    tops = np.array([0x00, 0x01, 0x65, 0x66, 0x67, 0x6E, 0x6F, 0x76, 0x77, 0x7E, 0x7E])
    for j in range(d_out):
        for b in range(0, d_in, OF.BLOCK):
            top, part = int(tops[rng.integers(len(tops))]), codes[j, b:b + OF.BLOCK]
            part[:] = (part & 0x80) | (part & 0x7F) % (top + 1)
            part[rng.integers(len(part))] = top | rng.integers(2) << 7
    return codes, scales


def encode(ck, ctx, codes, scales, block_rows, limbs, scale, bad=None, rounded=None):
    d_out, d_in = codes.shape
    enc = ck.empty_workspace(ck.ckks_fp8_weight_bytes(ctx, d_out, d_in, limbs))
    enc.fill_(-1)
    ck.ckks_linear_encode_fp8_units(ctx, ck.to_device(codes), ck.to_device(scales), d_out, d_in, block_rows, limbs, scale, enc,
                                    bad, rounded)
    return enc


def ints(a):
    import torch
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def check(ck, log_n, limbs, d_out, d_in, seed, block_rows=128, scale=2.0 ** 33):
    ctx = ctx_for(ck, log_n, limbs)
    codes, scales = spread_layer(seed, d_out, d_in, block_rows)
    ct = gen.uniform_residues(np.random.default_rng(seed + 1), (d_in, 2), ctx.moduli, ctx.n)
    bad, rounded = ints([3]), ints([4])
    enc = encode(ck, ctx, codes, scales, block_rows, limbs, scale, bad, rounded)
    assert int(bad) == 0 and int(rounded) == OF.rounded(codes)
    out = ck.empty_u32((d_out, 2, limbs, ctx.n))
    out.fill_(-1)
    ck.ckks_linear_mac_fp8(ctx, enc, ck.to_device(ct), out, d_out, d_in, limbs)
    cols = [0, 31, 32, 100, ctx.n - 1]
    got = ck.to_host_u32(out)
    want = OF.mac(codes, scales, ct[..., cols], block_rows, scale, ctx.moduli, in_units=True).astype(np.uint32)
    assert np.array_equal(got[..., cols], want)
    assert np.all(got < np.array(ctx.moduli, np.uint32)[None, None, :, None])


@gpu
@pytest.mark.parametrize("d_out,d_in", [(1, 1), (9, 128), (40, 33), (130, 127), (3, 129), (18, 700), (70, 300), (33, 1025)])
@pytest.mark.parametrize("block_rows", [1, 32, 128])
def test_sizes(gpu_lib, d_out, d_in, block_rows):
    check(gpu_lib, 10, 2, d_out, d_in, 800 + d_in, block_rows)


@gpu
@pytest.mark.parametrize("d_out,d_in", [(300, 40), (6, 600), (257, 320), (290, 640), (260, 1300)])
def test_every_kernel_of_many_columns(gpu_lib, d_out, d_in):
    check(gpu_lib, 10, MANY, d_out, d_in, 820 + d_in)


@gpu
def test_every_code_alone_is_kept(gpu_lib):
    """A row of one code has the unit of its own size: 512ths up to 56, and nothing is rounded."""
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    codes = np.arange(256, dtype=np.uint8).reshape(256, 1)
    ct = gen.uniform_residues(np.random.default_rng(1), (1, 2), ctx.moduli, ctx.n)
    scales = np.ones((2, 1), np.float32)
    bad, rounded = ints([9]), ints([9])
    enc = encode(ck, ctx, codes, scales, 128, 2, 512.0 * 12345, bad, rounded)
    assert int(bad) == 2 and int(rounded) == 0     # the two NaN
    out = ck.empty_u32((256, 2, 2, ctx.n))
    ck.ckks_linear_mac_fp8(ctx, enc, ck.to_device(ct), out, 256, 1, 2)
    f = np.nan_to_num(OF.numbers(codes[:, 0]), nan=0.0)
    exact = (f * 512).astype(np.int64) * 12345      # 512 12345 f, as rint(u f) rint(512 12345 / u) has to be
    want = np.stack([exact[:, None, None] % q * ct[0][None, :, l].astype(np.int64) % q for l, q in enumerate(ctx.moduli)], axis=2)
    assert np.array_equal(ck.to_host_u32(out), want.astype(np.uint32))


@gpu
def test_large_rows_are_encoded_as_in_64ths(gpu_lib):
    """The same bytes of a block where every row has a number past 224: the first two of three (columns 0 and 100, and
    200); fragments are [tile][step][2048 bytes], constants [limb][tile][block][384 bytes]."""
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 3)
    codes, scales = layer(840, 70, 300)
    codes[:, ::100] = 0x7D
    assert np.all(OF.units(codes)[:, :2] == 64) and np.any(OF.units(codes)[:, 2] != 64)
    same = []
    for enc in (encode(ck, ctx, codes, scales, 128, 3, 2.0 ** 30), encode_64ths(ck, ctx, codes, scales, 128, 3, 2.0 ** 30)):
        raw = enc.contiguous().cpu().numpy().view(np.uint8).reshape(-1)
        cut = 3 * 10 * 2048
        same.append((raw[:cut].reshape(3, 10, 2048)[:, :8], raw[cut:].reshape(3, 3, 3, 384)[:, :, :2]))
    assert np.array_equal(same[0][0], same[1][0]) and np.array_equal(same[0][1], same[1][1])


@gpu
def test_rows_much_smaller_than_their_block(gpu_lib):
    """What the encoding is for, through the product: inputs that are one-hot, so that outputs are the plaintexts.  Rows spread over
    1 : 10^4 in one block: each weight within 1 / 28672 of its row's largest and a 512th's share of its scale."""
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    rng = np.random.default_rng(845)
    w = rng.normal(0, 0.02, (64, 128)) * np.geomspace(1, 1e-4, 64)[:, None]
    s = np.float32(np.abs(w).max() / 448)
    import torch
    w8 = torch.from_numpy(w / s).to(torch.float8_e4m3fn)
    codes, delta = w8.view(torch.uint8).numpy(), 2.0 ** 36
    scales = np.full((1, 1), s, np.float32)
    ct = np.zeros((128, 2, 2, ctx.n), np.uint32)
    ct[np.arange(128), 0, :, np.arange(128)] = 1
    off = {}
    for name, enc in (("units", encode(ck, ctx, codes, scales, 128, 2, delta)), ("64ths", encode_64ths(ck, ctx, codes, scales, 128, 2, delta))):
        out = ck.empty_u32((64, 2, 2, ctx.n))
        ck.ckks_linear_mac_fp8(ctx, enc, ck.to_device(ct), out, 64, 128, 2)
        r = ck.to_host_u32(out)[:, 0, :, :128].astype(object)
        q0, q1 = ctx.moduli
        x = r[:, 0] + q0 * ((r[:, 1] - r[:, 0]) * pow(q0, -1, q1) % q1)
        got = np.where(x > q0 * q1 // 2, x - q0 * q1, x).astype(np.float64) / delta
        true = OF.numbers(codes) * float(s)
        off[name] = np.abs(got - true)
        top = np.abs(true).max(axis=1, keepdims=True)
        if name == "units":
            assert np.all(off[name] <= top / 28672 + np.abs(true) * 512 / (2 * float(s) * delta) * (1 + 2.0 ** -20))
    assert (off["64ths"] / top).max() > 0.1       # the form without units loses a small row


@gpu
def test_what_is_no_number_is_counted(gpu_lib):
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    codes, scales = spread_layer(850, 300, 200, 64)
    codes[0, 0] = codes[299, 199] = codes[64, 128] = 0x7F
    codes[100, :] = 0xFF                                            # a row of nothing else
    scales[0, 1], scales[4, 0], scales[2, 0], scales[3, 1] = np.inf, np.nan, -np.inf, 0.0
    scales[1, 0], scales[1, 1] = 256 / 2.0 ** 33, 257 / 2.0 ** 33   # half of a 512th's unit goes to zero, a little more does not
    bad, rounded = ints([77]), ints([78])
    for _ in range(2):
        enc = encode(ck, ctx, codes, scales, 64, 2, 2.0 ** 33, bad, rounded)
        assert int(bad) == 3 + 200 + 3 + 1 and int(rounded) == OF.rounded(codes)
    ct = gen.uniform_residues(np.random.default_rng(851), (200, 2), ctx.moduli, ctx.n)
    out = ck.empty_u32((300, 2, 2, ctx.n))
    ck.ckks_linear_mac_fp8(ctx, enc, ck.to_device(ct), out, 300, 200, 2)
    assert np.array_equal(ck.to_host_u32(out), OF.mac(codes, scales, ct, 64, 2.0 ** 33, ctx.moduli, in_units=True).astype(np.uint32))


@gpu
@pytest.mark.parametrize("encoder", [encode, encode_64ths])
def test_scales_that_vanish_in_fp64_are_counted(gpu_lib, encoder):
    """1e-30 * 1e-300 is zero in fp64 already, before anything is rounded; a zero times it is no loss."""
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 1)
    codes, _ = layer(855, 5, 300)
    bad = ints([0])
    encoder(ck, ctx, codes, np.array([[1e-30, 0.0, -1e-40]], np.float32), 128, 1, 1e-300, bad)
    assert int(bad) == 2


@gpu
def test_experts_on_another_stream_and_in_a_graph(gpu_lib):
    """Two experts, one of each encoding, from weights at an odd address."""
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 11, 2)
    d_out, d_in = 66, 129
    codes, scales = spread_layer(860, d_out, d_in, 64)
    ct = gen.uniform_residues(np.random.default_rng(861), (2, d_in, 2), ctx.moduli, ctx.n)
    want = np.stack([OF.mac(codes, scales, ct[1], 64, 2.0 ** 33, ctx.moduli, in_units=u).astype(np.uint32) for u in (False, True)])
    w8 = torch.empty(codes.size + 1, dtype=torch.uint8, device="cuda")[1:].view(codes.shape)
    w8.copy_(torch.from_numpy(codes))
    d_s, d_ct = ck.to_device(scales), ck.to_device(ct)
    enc = ck.empty_workspace(2 * ck.ckks_fp8_weight_bytes(ctx, d_out, d_in, 2)).view(2, -1)
    bad, rounded = ints([0]), ints([0])
    out = ck.empty_u32((2, d_out, 2, 2, ctx.n))
    expert, bundle = ints([0, 1]), ints([1, 1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def calls():
        ck.ckks_linear_encode_fp8(ctx, w8, d_s, d_out, d_in, 64, 2, 2.0 ** 33, enc[0], stream=s)
        ck.ckks_linear_encode_fp8_units(ctx, w8.view(torch.float8_e4m3fn), d_s, d_out, d_in, 64, 2, 2.0 ** 33, enc[1], bad, rounded, stream=s)
        ck.ckks_experts_mac_fp8(ctx, enc, expert, bundle, d_ct, out, d_out, d_in, 2, stream=s)
    with torch.cuda.stream(s):
        calls()
    s.synchronize()
    assert np.array_equal(ck.to_host_u32(out), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        calls()
    for _ in range(3):
        out.fill_(0)
        enc.fill_(-1)
        rounded.fill_(9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(ck.to_host_u32(out), want) and int(bad) == 0 and int(rounded) == OF.rounded(codes)
    del graph


@gpu
def test_empty_layers_and_refusals(gpu_lib):
    import torch
    ck = gpu_lib
    ctx = ctx_for(ck, 10, 2)
    bad, rounded = ints([5]), ints([6])
    ck.ckks_linear_encode_fp8_units(ctx, None, None, 0, 5, 128, 2, 1.0, None, bad, rounded)
    assert int(bad) == 0 and int(rounded) == 0
    codes, scales = layer(870, 16, 64)
    w8, d_s = ck.to_device(codes), ck.to_device(scales)
    enc = ck.empty_workspace(ck.ckks_fp8_weight_bytes(ctx, 16, 64, 2))
    raw, wrong = ck._lib.ckks_linear_encode_fp8_units, ck.CKKS_E_INVALID_ARG

    def call(w=w8.data_ptr(), s=d_s.data_ptr(), rows=128, limbs=2, scale=1.0, to=enc.data_ptr(), b=bad.data_ptr(), r=rounded.data_ptr()):
        return raw(ctx.handle, w, s, 16, 64, rows, limbs, scale, to, b, r, None)
    for args in (dict(w=None), dict(s=None), dict(rows=0), dict(limbs=3), dict(scale=0.0), dict(scale=float("nan")), dict(to=None),
                 dict(to=enc.data_ptr() + 8), dict(s=d_s.data_ptr() + 2), dict(b=bad.data_ptr() + 1), dict(r=rounded.data_ptr() + 2),
                 dict(r=bad.data_ptr()), dict(r=enc.data_ptr() + 4), dict(r=d_s.data_ptr()), dict(w=enc.data_ptr())):
        assert call(**args) == wrong, args
        assert ck.ckks_last_error()
    for other in (bad.float(), bad.to(torch.int64)):
        with pytest.raises(ValueError, match="rounded must be int32"):
            ck.ckks_linear_encode_fp8_units(ctx, w8, d_s, 16, 64, 128, 2, 1.0, enc, bad, other)
    with pytest.raises(ValueError):
        ck.ckks_linear_encode_fp8_units(ctx, w8.view(torch.int8), d_s, 16, 64, 128, 2, 1.0, enc)
    with pytest.raises(ValueError):
        ck.ckks_linear_encode_fp8_units(ctx, w8, d_s, 16, 64, 1, 2, 1.0, enc)


def test_null_context_is_rejected_without_a_gpu():
    import paper_2606_17421_amd as ck
    assert ck._lib.ckks_linear_encode_fp8_units(None, None, None, 1, 1, 128, 1, 1.0, None, None, None, None) == ck.CKKS_E_INVALID_ARG
