"""CPU checks of how the attention's work is divided: the library's own header, compiled on the spot."""
import ctypes
import os
import subprocess

import pytest

SHIM = """
#include "ivfpq_attention_rules.hpp"
extern "C" void plan(long long n, int m, int heads, int kv_heads, int d, long long places, int* out) {
    const ivfpq::AttentionPlan p = ivfpq::attention_plan(n, m, heads, kv_heads, d, places);
    out[0] = p.tiles, out[1] = p.apart, out[2] = p.blocks, out[3] = p.parts, out[4] = p.columns(), out[5] = p.waves;
}
extern "C" long long scratch(long long n, int m, int heads, int kv_heads, int d, long long places) {
    return ivfpq::attention_scratch_bytes(n, kv_heads, d, ivfpq::attention_plan(n, m, heads, kv_heads, d, places));
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    where = tmp_path_factory.mktemp("rules")
    (where / "shim.cpp").write_text(SHIM)
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2301_06672_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", csrc, str(where / "shim.cpp"), "-o", str(where / "shim.so")], check=True)
    lib = ctypes.CDLL(str(where / "shim.so"))
    lib.plan.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_longlong, ctypes.POINTER(ctypes.c_int)]
    lib.scratch.argtypes = lib.plan.argtypes[:-1]
    lib.scratch.restype = ctypes.c_longlong

    def ask(*args):
        out = (ctypes.c_int * 6)()
        lib.plan(*args, out)
        return dict(zip(("tiles", "apart", "blocks", "parts", "columns", "waves"), out))
    ask.scratch = lib.scratch
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
            assert got["tiles"] in (1, 2) and not (d > 128 and got["tiles"] == 2) and got["waves"] in (4, 8)
            assert got["columns"] * got["blocks"] >= m * share > got["columns"] * (got["blocks"] - 1)
            assert got["parts"] == 0 or n < got["parts"] <= 64 * n
            # workgroups that share a wave's columns have one block of them: they divide the places, and add up in the LDS
            assert got["apart"] or got["blocks"] == 1


def test_places_are_divided_where_workgroups_are_few(plan):
    assert plan(1, 1, 32, 8, 128, 100)["parts"] == 0                     # too short
    assert plan(1, 1, 32, 8, 128, 100_000)["parts"] == 64
    assert plan(16, 64, 32, 8, 128, 8_192)["parts"] == 48                # two rounds of pieces, 8 x (48 + 16)
    assert plan(1_000, 1, 32, 8, 128, 100_000)["parts"] == 0             # workgroups enough
    assert plan.scratch(1_000, 1, 32, 8, 128, 100_000) == 0
    assert plan.scratch(16, 64, 32, 8, 128, 8_192) == 8 * (48 + 16) * 256 * 130 * 4 + 16 * 8
