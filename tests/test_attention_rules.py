"""CPU checks of how the attention's work is divided: the library's own header, compiled on the spot."""
import ctypes
import os
import subprocess

import pytest

SHIM = """
#include "ivfpq_attention_rules.hpp"
extern "C" void plan(long long n, int m, int heads, int kv_heads, int d, long long places, int* out) {
    const ivfpq::AttentionPlan p = ivfpq::attention_plan(n, m, heads, kv_heads, d, places);
    out[0] = p.tiles, out[1] = p.apart, out[2] = p.blocks, out[3] = p.splits, out[4] = p.columns();
}
extern "C" long long floats(long long n, int m, int heads, int d, int splits) { return ivfpq::attention_split_floats(n, m, heads, d, splits); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    where = tmp_path_factory.mktemp("rules")
    (where / "shim.cpp").write_text(SHIM)
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2301_06672_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", csrc, str(where / "shim.cpp"), "-o", str(where / "shim.so")], check=True)
    lib = ctypes.CDLL(str(where / "shim.so"))
    lib.plan.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_longlong, ctypes.POINTER(ctypes.c_int)]
    lib.floats.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int]
    lib.floats.restype = ctypes.c_longlong

    def ask(*args):
        out = (ctypes.c_int * 5)()
        lib.plan(*args, out)
        return dict(zip(("tiles", "apart", "blocks", "splits", "columns"), out))
    ask.floats = lib.floats
    return ask


@pytest.mark.parametrize("d", [8, 64, 128, 136, 256])
@pytest.mark.parametrize("share", [1, 3, 8, 64])
@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 64, 65, 1000, 1 << 20])
def test_every_column_has_a_place(plan, d, share, m):
    for n, kv_heads in ((1, 1), (7, 8)):
        if n * m * share * kv_heads > 1 << 26:
            continue
        for places in (0, 1, 127, 4_096, 2 ** 31 - 2 ** 21):
            got = plan(n, m, share * kv_heads, kv_heads, d, places)
            assert got["tiles"] in (1, 2, 4) and not (d > 128 and got["tiles"] == 4)
            assert got["columns"] * got["blocks"] >= m * share > got["columns"] * (got["blocks"] - 1)
            assert 1 <= got["splits"] <= 64
            # workgroups that share a wave's columns have one block of them: they divide the places, and add up in the LDS
            assert got["apart"] or got["blocks"] == 1


def test_places_are_divided_where_workgroups_are_few(plan):
    assert plan(1, 1, 32, 8, 128, 100)["splits"] == 1                    # too short
    assert plan(1, 1, 32, 8, 128, 100_000)["splits"] > 8
    assert plan(1_000, 1, 32, 8, 128, 100_000)["splits"] == 1            # workgroups enough
    assert plan.floats(3, 5, 8, 64, 1) == 0 and plan.floats(3, 5, 8, 64, 4) == 3 * 5 * 8 * 4 * 66
