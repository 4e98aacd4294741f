"""The encrypted K/V example: projections over 4-bit weights, the paged cache's
calls and the decryption through its table, run together as a server runs them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

EXAMPLE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "encrypted_kv.py")


def test_encrypted_kv_example(gpu_lib):
    spec = importlib.util.spec_from_file_location("encrypted_kv", EXAMPLE)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    out = mod.main(seed=7)
    assert out["status"] == [0, 0]
    # 6 prompt rows on 2 pages; both continuations copy the second page's 2 rows; the prompt's copy of it is freed
    assert (out["held_before"], out["held_after"]) == (4, 3)
    assert out["rows"] == 14
    # 2 * 7 * 32 * 512 slots: 6 standard deviations of the rescale's rounding, of which the encryption and
    # encoding errors (3.2 sqrt(N/2) sum|W| / 2^50 and below) are less than a hundredth
    assert out["worst_over_sd"] <= 6
