"""CPU checks of the rules that choose the kernels of the language-model calls: the library's own header, compiled on the spot."""
import ctypes
import os
import subprocess

import pytest

import util_products

SHIM = """
#include "ivfpq_language_rules.hpp"
extern "C" int product(long long m, long long n, int k, int* rows, int* columns) {
    const ivfpq::ProductKernel c = ivfpq::product_kernel(m, n, k);
    *rows = c.rows;
    *columns = c.columns;
    return c.tiles;
}
extern "C" int in_registers(long long n, long long vocab, int value_bytes) { return ivfpq::step_in_registers(n, vocab, value_bytes); }
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    where = tmp_path_factory.mktemp("rules")
    (where / "shim.cpp").write_text(SHIM)
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2301_06672_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", csrc, str(where / "shim.cpp"), "-o", str(where / "shim.so")], check=True)
    lib = ctypes.CDLL(str(where / "shim.so"))
    lib.product.argtypes = [ctypes.c_longlong, ctypes.c_longlong, ctypes.c_int] + [ctypes.POINTER(ctypes.c_int)] * 2
    lib.in_registers.argtypes = [ctypes.c_longlong, ctypes.c_longlong, ctypes.c_int]
    return lib


def product(rules, m, n, k):
    rows, columns = ctypes.c_int(), ctypes.c_int()
    tiles = rules.product(m, n, k, rows, columns)
    return bool(tiles), rows.value, columns.value


def test_products_that_were_measured(rules):
    # the faster side of every figure at the rule
    for m, n, k, tiles, rows in [(32, 4000, 4096, False, 32), (32, 16000, 4096, False, 32), (32, 32768, 4096, True, 128), (64, 8000, 4096, False, 64),
                                 (64, 32768, 4096, True, 128), (1000, 30000, 900, True, 256), (512, 32768, 4096, True, 256), (777, 100003, 96, True, 128),
                                 (1, 32768, 4096, False, 16), (2048, 32768, 4096, True, 256)]:
        assert product(rules, m, n, k)[:2] == (tiles, rows), (m, n, k)
    assert product(rules, 32, 4000, 4096)[2] == 16 and product(rules, 16, 32768, 4096)[2] == 32


def test_sizes_of_the_tests_of_tiles_take_tiles(rules):
    for m, n, k, tile, aligned in util_products.TILES:
        assert product(rules, m, n, k) == (True, tile, tile), (m, n, k)
        assert aligned == (4 * n % 64 == 0, 2 * n % 64 == 0)
    for m, n, k, tile in util_products.LAYOUTS:
        assert product(rules, m, n, k) == (True, tile, tile), (m, n, k)
    for far, m, n, k, tile in util_products.FAR:
        assert product(rules, m, n, k) == (True, tile, tile), (m, n, k)
        assert (m if far == "a" else n) >= tile


@pytest.mark.parametrize("m", [1, 16, 17, 32, 33, 64, 65, 4096, 1 << 22])
@pytest.mark.parametrize("n", [1, 16, 8191, 8192, 40000, 1 << 22])
def test_strips_have_a_launch(rules, m, n):
    """A grid's second dimension ends at 65,535."""
    tiles, rows, columns = product(rules, m, n, 64)
    assert tiles or (-(-m // rows) <= 65535 and rows in (16, 32, 64) and columns in (16, 32))


# distillation steps, us: rows, values, bytes of one; called one after the other, replayed from a graph, in registers and split each
STEPS = [(1, 50000, 2, 13.8, 19.1, 12.0, 12.0), (64, 50000, 2, 15.8, 19.0, 16.2, 17.8), (160, 50000, 2, 20.7, 25.5, 21.1, 25.8), (8, 65536, 2, 14.5, 19.2, 14.6, 13.1),
         (32, 65536, 2, 17.1, 19.1, 17.3, 17.5), (160, 65536, 2, 23.6, 27.1, 23.6, 27.4), (1, 80000, 2, 15.8, 18.9, 15.6, 11.9), (24, 80000, 2, 18.4, 19.1, 18.5, 16.6),
         (96, 80000, 2, 23.1, 25.0, 23.5, 25.3), (16, 100000, 2, 21.1, 19.2, 21.2, 16.4), (48, 100000, 2, 24.6, 19.6, 25.3, 20.0), (96, 100000, 2, 26.9, 25.6, 27.2, 26.0),
         (128, 100000, 2, 27.6, 29.2, 27.8, 29.7), (1, 131072, 2, 24.0, 18.8, 23.5, 12.4), (16, 131072, 2, 24.9, 19.0, 25.3, 16.3), (32, 131072, 2, 26.5, 19.1, 27.6, 19.4),
         (64, 131072, 2, 30.4, 25.3, 30.7, 25.5), (96, 131072, 2, 32.3, 28.8, 32.5, 29.0), (128, 131072, 2, 32.4, 33.8, 32.8, 34.2), (160, 131072, 2, 34.3, 39.1, 34.9, 39.7),
         (1, 50000, 4, 13.6, 18.8, 11.0, 11.5), (16, 65536, 4, 13.8, 19.2, 13.3, 15.6), (160, 65536, 4, 24.9, 38.0, 25.2, 38.6)]


@pytest.mark.parametrize("n,vocab,size,called,called_split,replayed,replayed_split", STEPS)
def test_steps_that_were_measured(rules, n, vocab, size, called, called_split, replayed, replayed_split):
    """The faster route where both ways of calling agree; elsewhere rows are split below 16 of them."""
    agree = (called < called_split) == (replayed <= replayed_split)
    assert bool(rules.in_registers(n, vocab, size)) == (called < called_split if agree else n >= 16)


def test_rows_that_no_registers_hold(rules):
    assert not rules.in_registers(4096, 131073, 2) and not rules.in_registers(4096, 65537, 4) and rules.in_registers(4096, 131072, 2)
