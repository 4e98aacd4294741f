"""Pins of the oracle's 8-bit layer: the numbers of e4m3, written-out cases, the
distance of a rounded weight, and the scalar route where both round alike."""
import numpy as np
import pytest

from oracle import encode, fp8, linear, params


def test_the_numbers_of_e4m3():
    at = {0x00: 0.0, 0x01: 2.0 ** -9, 0x07: 7 * 2.0 ** -9, 0x08: 2.0 ** -6, 0x38: 1.0, 0x39: 1.125, 0x7E: 448.0, 0xFE: -448.0,
          0xB8: -1.0, 0x40: 2.0}
    assert {c: float(fp8.numbers([c])[0]) for c in at} == at
    assert np.isnan(fp8.numbers([0x7F, 0xFF])).all()


def test_the_numbers_are_torchs():
    import torch
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(fp8.numbers(codes.numpy()), want, equal_nan=True)


def test_a_written_out_layer():
    # 448, -1, 5/512 (rounds to 1/64), 4/512 = half a 64th (to even: 0) and 12/512 (to even: 2/64)
    codes = np.array([[0x7E, 0xB8, 0x05, 0x04, 0x0C], [0x38, 0x7F, 0x00, 0x80, 0xFE]], np.uint8)
    p = fp8.plaintexts(codes, np.array([[0.5], [-0.25]], np.float32), 1, 64 * 8.0)
    assert p.tolist() == [[28672 * 4, -64 * 4, 4, 0, 2 * 4], [64 * -2, 0, 0, 0, 28672 * 2]]


def test_blocks_and_scales():
    codes = np.full((5, 130), 0x38, np.uint8)
    scales = np.array([[0.5, 1.5], [np.inf, np.nan], [2.5, -2.5]], np.float32)   # halves round to even; no number is zero
    p = fp8.plaintexts(codes, scales, 2, 64.0)
    assert p[:, 0].tolist() == [0, 0, 0, 0, 64 * 2] and p[:, 129].tolist() == [64 * 2, 64 * 2, 0, 0, 64 * -2]
    assert fp8.plaintexts(codes[:1, :1], [[1.0]], 1, 2.0 ** 68)[0, 0] == 64 << 62


def test_distance_to_the_weights():
    """From 1/8 on a number is a multiple of 1/64, below it within half of one."""
    f = fp8.numbers([c for c in range(256) if c & 0x7F != 0x7F])
    far = np.abs(np.rint(64 * f) / 64 - f)
    assert far[np.abs(f) >= 0.125].max() == 0 and far.max() == 2.0 ** -7


def test_a_written_out_layer_in_units():
    # rows whose largest are 56, 60, 120, 240 and 0: units 512, 256, 128, 64 and 512; 5/512 beside each
    codes = np.array([[0x66, 0x05], [0x67, 0x05], [0x6F, 0x05], [0x77, 0x85], [0x7F, 0x80]], np.uint8)
    assert fp8.numbers(codes)[:4, 0].tolist() == [56, 60, 120, 240]
    assert fp8.units(codes)[:, 0].tolist() == [512, 256, 128, 64, 512]
    p = fp8.plaintexts_in_units(codes, np.array([[1.0]], np.float32), 128, 512.0 * 3)
    # 2.5 of 256ths and 1.25, 0.625 of the coarser ones round to 2, 1 and 1
    assert p.tolist() == [[28672 * 3, 5 * 3], [15360 * 6, 2 * 6], [15360 * 12, 12], [15360 * 24, -24], [0, 0]]
    assert fp8.rounded(codes) == 3


def test_scales_that_vanish_in_512ths_are_zero():
    codes = np.array([[0x38], [0x7E]], np.uint8)
    for size, want in ((256.0, [0, 0]), (257.0, [512, 28672 * 4])):
        assert fp8.plaintexts_in_units(codes, np.array([[1.0]], np.float32), 128, size)[:, 0].tolist() == want


def test_distance_to_small_rows():
    """Each weight within 1 / 28672 of its row's largest, whatever else is in the block, and kept where that is up to 56."""
    rng = np.random.default_rng(6)
    f = rng.normal(0, 100, (128, 128)) * np.geomspace(1, 1e-4, 128)[:, None]
    import torch
    codes = torch.from_numpy(f).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    f, u = fp8.numbers(codes), fp8.units(codes)
    top = np.abs(f).max(axis=1, keepdims=True)
    far = np.abs(np.rint(u * f) / u - f)
    assert np.all(far <= top / 28672) and np.all(far[top[:, 0] <= 56] == 0) and set(u[:, 0]) == {64, 128, 256, 512}


@pytest.mark.parametrize("block_rows", [1, 3, 128])
def test_mac_is_the_scalar_mac_where_the_scales_are_exact(block_rows):
    rng = np.random.default_rng(4)
    qs = params.moduli(10, 2)
    codes = rng.choice([c for c in range(256) if 0x20 <= c & 0x7F < 0x7F], (5, 200)).astype(np.uint8)   # 1/8 and above
    scales = (rng.integers(-1000, 1000, (-(-5 // block_rows), 2)) / 1024.0).astype(np.float32)
    ct = np.stack([rng.integers(0, q, (200, 2, 16)) for q in qs], axis=2).astype(np.uint32)
    w = fp8.numbers(codes) * scales.astype(np.float64)[np.arange(5) // block_rows][:, np.arange(200) // 128]
    want = linear.mac_scalar(encode.encode_scalar(w, 2.0 ** 20, qs), ct, qs)
    assert np.array_equal(fp8.mac(codes, scales, ct, block_rows, 2.0 ** 20, qs), want)


def test_combine_is_the_polynomial_mac():
    """One feature: the sum over a bundle's terms is a row of the full-polynomial MAC."""
    rng = np.random.default_rng(5)
    qs = params.moduli(10, 2)
    draw = lambda *s: np.stack([rng.integers(0, q, s + (8,)) for q in qs], axis=-2).astype(np.uint32)  # noqa: E731
    gates, y = draw(3), draw(3, 1, 2)
    got = fp8.combine(gates, y, [[0, 2, -1], [1, 1, 3], [-1, -5, 3]], qs)
    want = linear.mac_poly(np.stack([gates[[0, 2]], gates[[1, 1]]]), y[[0, 2], 0], qs)
    assert np.array_equal(got[0, 0], want[0])
    twice = linear.mac_poly(gates[[1, 1]][None], y[[1, 1], 0], qs)
    assert np.array_equal(got[1, 0], twice[0]) and not got[2].any()
