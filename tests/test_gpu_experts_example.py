"""The encrypted mixture-of-experts example: encryption, the experts' products over
8-bit weights, rescale, the gated sums, rescale and decryption, as a server runs them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

EXAMPLE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "encrypted_experts.py")


def test_encrypted_experts_example(gpu_lib):
    spec = importlib.util.spec_from_file_location("encrypted_experts", EXAMPLE)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    out = mod.main(seed=7)
    assert out["requests"] == 7                      # four experts of the first bundle, three of the second
    assert out["status"] == [0] * 7 + [1] * 3
    # 2 * 40 * 512 slots within six standard deviations of the sum of all roundings and errors
    assert out["worst_over_sd"] <= 6
    assert out["largest"] > 1000 * out["worst_error"]


def test_encrypted_experts_example_against_the_quantised_weights(gpu_lib):
    """The decrypted layer against scales times e4m3 numbers: an error of the encoding itself, which the comparison with the
    encoded weights cannot show, is within the rounding that the header states."""
    spec = importlib.util.spec_from_file_location("encrypted_experts", EXAMPLE)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    out = mod.main(seed=8)
    assert out["worst_from_layer"] <= 1
    # the bound says something: 200 weights off by 28672 / 2^32 for their scale and s / 128 for their size (s = 0.02 * 5 / 448 at
    # most) are 1.7e-3, and the largest output, 0.58 * 0.02 * sqrt(200) = 0.16 times more than 2, is over 0.3
    assert out["largest_rounding"] < 1.7e-3 and out["largest"] > 0.3
