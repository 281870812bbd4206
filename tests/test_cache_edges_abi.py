"""More of what the paged cache's entry points refuse, and of the binding's own arithmetic.  No
GPU."""
import pytest

from test_abi import FAKE, lib  # noqa: F401  (lib: fixture)
from test_cache_abi import Decode, Write


@pytest.mark.parametrize("make", [Write, Decode])
@pytest.mark.parametrize("off", [4, 8, 12])
def test_misaligned_key_sums(lib, make, off):  # noqa: F811
    c = make()
    c.c.t["k_sum"].data = FAKE + off
    assert c.call(lib) == "MOBA_ERR_LAYOUT"
