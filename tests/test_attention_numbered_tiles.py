"""CPU check of which page tables' tiles can be dealt to parts: the library's own header, compiled on the spot."""
import ctypes
import os
import subprocess

import pytest

SHIM = """
#include "ivfpq_attention_rules.hpp"
extern "C" int numbered(long long n, long long places) { return ivfpq::tiles_numbered(n, places); }
extern "C" int parts(long long n, int m, int heads, int kv_heads, int d, long long places) { return ivfpq::attention_plan(n, m, heads, kv_heads, d, places).parts; }
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    where = tmp_path_factory.mktemp("numbered")
    (where / "shim.cpp").write_text(SHIM)
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2301_06672_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", csrc, str(where / "shim.cpp"), "-o", str(where / "shim.so")], check=True)
    lib = ctypes.CDLL(str(where / "shim.so"))
    lib.numbered.argtypes = [ctypes.c_longlong, ctypes.c_longlong]
    lib.parts.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_longlong]
    return lib


@pytest.mark.parametrize("n", [1, 31, 32, 33, 40, 1 << 20])
@pytest.mark.parametrize("page", [16, 256])
def test_tiles_fit_31_bits(rules, n, page):
    """A sequence of p places has up to p / 32 + 1 tiles, and one where it has none; the kernel numbers all of them, from 0, in an int32."""
    for places in (0, page, 10 ** 6, 2 ** 31 * 32 // n // page * page - page, 2 ** 31 * 32 // n // page * page + page, 2 ** 31 - 2 ** 21 - page):
        if not 0 <= places < 2 ** 31 - 2 ** 21:
            continue
        if rules.numbered(n, places):
            assert n * max(-(-places // 32), 1) < 2 ** 31
        else:
            assert n * (places // 32 + 2) >= 2 ** 31


def test_any_bound_gives_a_plan(rules):
    """max_places may be anything: a plan divides, or does not, whatever the table."""
    assert rules.parts(4, 1, 8, 2, 128, 0) == 0
    assert rules.parts(64, 1, 1, 1, 128, 2 ** 31 - 2 ** 21) > 64
