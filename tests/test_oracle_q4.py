"""Pins of the oracle's 4-bit layer: written-out cases, the nibble order, and the
scalar route where both round alike."""
import numpy as np
import pytest

from oracle import encode, linear, params, q4


def test_a_written_out_layer():
    # two inputs share a scale, a third has its own; u = 0 and 15 are the ends
    w4 = np.array([[0xF0, 0x09]], np.uint8)            # u = 0, 15, 9
    scales = np.array([[0.5, -0.25]], np.float32)
    p = q4.plaintexts(w4, scales, None, 3, 2, 8.0)
    assert p.tolist() == [[-8 * 4, 7 * 4, 1 * -2]]
    p = q4.plaintexts(w4, scales, np.array([[15, 0x40]], np.uint8), 3, 2, 8.0)  # only four bits of a zero point count
    assert p.tolist() == [[-15 * 4, 0, 9 * -2]]


def test_scales_round_half_to_even():
    w4 = q4.pack([[9, 9, 9]])
    p = q4.plaintexts(w4, np.array([[0.5, 1.5, -2.5]], np.float32), None, 3, 1, 1.0)
    assert p.tolist() == [[0, 2, -2]]


@pytest.mark.parametrize("d_in", [1, 2, 5, 8])
def test_pack_and_unpack(d_in):
    u = np.random.default_rng(d_in).integers(0, 16, (3, d_in))
    w4 = q4.pack(u)
    assert w4.shape == (3, (d_in + 1) // 2)
    assert np.array_equal(q4.unpack(w4, d_in), u)


@pytest.mark.parametrize("zeros", [False, True])
def test_mac_is_the_scalar_mac_where_the_scales_are_exact(zeros):
    rng = np.random.default_rng(4)
    qs = params.moduli(10, 2)
    u, z = rng.integers(0, 16, (5, 70)), rng.integers(0, 16, (5, 3))
    scales = (rng.integers(-1000, 1000, (5, 3)) / 1024.0).astype(np.float32)
    ct = np.stack([rng.integers(0, q, (70, 2, 16)) for q in qs], axis=2).astype(np.uint32)
    of = np.arange(70) // 32
    w = (u - (z[:, of] if zeros else 8)) * scales.astype(np.float64)[:, of]
    want = linear.mac_scalar(encode.encode_scalar(w, 2.0 ** 20, qs), ct, qs)
    got = q4.mac(q4.pack(u), scales, z if zeros else None, ct, 32, 2.0 ** 20, qs)
    assert np.array_equal(got, want)


def test_scales_beyond_a_prime():
    qs = params.moduli(10, 1)
    p = q4.plaintexts(q4.pack([[15]]), np.array([[1.0]], np.float32), None, 1, 32, 2.0 ** 62)
    assert p[0, 0] == 7 << 62
    assert q4.residues(p, qs)[0, 0, 0] == (7 << 62) % qs[0]


@pytest.mark.parametrize("zeros,from_product,from_rounding", [(True, 7.5, 8), (False, 4, 4)])
def test_distance_to_the_rounded_products(zeros, from_product, from_rounding):
    """The scale is rounded before the product: at most half a unit times the small integer, and a
    rounding more; scaled scales of halves reach both."""
    u = np.arange(16).reshape(16, 1)
    far = [0.0, 0.0]
    for z in range(16) if zeros else (8,):
        for s in (0.5, 1.5, 2.49, 0.25, 1000.5):
            p = q4.plaintexts(q4.pack(u), np.full((16, 1), s, np.float32), np.full((16, 1), z, np.uint8) if zeros else None,
                              1, 32, 1.0).astype(float)
            product = (u - z) * np.float64(np.float32(s))
            far = [max(far[0], abs(p - product).max()), max(far[1], abs(p - np.rint(product)).max())]
    assert far == [from_product, from_rounding]
