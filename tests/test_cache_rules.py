"""The paged cache's arithmetic on lengths (csrc/cache_rules.h, compiled for the host), up to the
longest that 32 bits hold."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = """
#include "cache_rules.h"
extern "C" int cache_steps(int len) { return moba::cache_steps(len); }
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "shim.cpp").write_text(SHIM)
    so = str(d / "shim.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2502_13189_amd", "csrc"), str(d / "shim.cpp"), "-o", so],
                   check=True)
    return ctypes.CDLL(so)


def test_steps(rules):
    top = 2 ** 31 - 1
    for n in (*range(200), 2 ** 24 - 1, 2 ** 24, *range(top - 200, top + 1)):
        assert rules.cache_steps(n) == -(-n // 64), n
