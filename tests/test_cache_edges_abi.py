"""More of what the paged cache's entry points refuse, and of the binding's own arithmetic.  No
GPU."""
import pytest

from paper_2502_13189_amd import binding
from test_abi import FAKE, lib  # noqa: F401  (lib: fixture)
from test_cache_abi import Decode, Write


@pytest.mark.parametrize("make", [Write, Decode])
@pytest.mark.parametrize("off", [4, 8, 12])
def test_misaligned_key_sums(lib, make, off):  # noqa: F811
    c = make()
    c.c.t["k_sum"].data = FAKE + off
    assert c.call(lib) == "MOBA_ERR_LAYOUT"


def test_workspace_bytes_of_what_passes_32_bits(lib):  # noqa: F811
    good = (3, 40, 8, 2, 128, 256, 3)
    assert binding.cache_decode_workspace_bytes(*good) > 0
    for i in range(6):  # (a call with such a size is refused)
        for more in (1 << 32, -(1 << 32), 1 << 64, 1 << 31):
            bad = list(good)
            bad[i] += more
            assert binding.cache_decode_workspace_bytes(*bad) == 0, bad
    # a topk past every block attends everything, however large
    assert binding.cache_decode_workspace_bytes(*good[:6], (1 << 32) + 3) == binding.cache_decode_workspace_bytes(
        *good[:6], 1000)
    assert binding.cache_decode_workspace_bytes(*good[:6], 3 - (1 << 32)) == 0
