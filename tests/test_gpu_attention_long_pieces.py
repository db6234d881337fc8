"""ivfpq_draft_attention where a workgroup goes over many tiles: what its loops carry from one step to the next (stages of the LDS that are written again, pages looked up
steps ahead, registers loaded ahead), the switch to masked tiles late in a piece, odd numbers of tiles, pieces joined.  Every test asserts by the library's own rules how
many steps its pieces have, so that other rules cannot shorten it unnoticed.

Half of the columns look for one place each, whose key they are a multiple of: their results are that place's values, so a tile that is missed, taken twice or
for another is off by about the values' size.  The places looked for are spread over all that a column sees.

Tolerance.  As for short pieces: half a step of the cache's type for the weights and for the result; scores of d products in fp32, whose error e changes weights by a factor
of exp(2 e) at most; weights of fp16 under 2^-30 of the largest cut off.  And sums over P places: up to P + 64 additions one after the other, each off by 2^-24 of
what the sum holds, in the numerator and in the denominator."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from util_drafts import Cache, half_step, tree

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16

SHIM = """
#include "ivfpq_attention_rules.hpp"
extern "C" void plan(long long n, int m, int heads, int kv_heads, int d, long long places, int* out) {
    const ivfpq::AttentionPlan p = ivfpq::attention_plan(n, m, heads, kv_heads, d, places);
    out[0] = p.apart, out[1] = p.waves, out[2] = p.columns(), out[3] = p.blocks, out[4] = p.parts;
}
"""


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    where = tmp_path_factory.mktemp("rules")
    (where / "shim.cpp").write_text(SHIM)
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2301_06672_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", csrc, str(where / "shim.cpp"), "-o", str(where / "shim.so")], check=True)
    lib = ctypes.CDLL(str(where / "shim.so"))
    lib.plan.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_longlong, ctypes.POINTER(ctypes.c_int)]

    def ask(*args):
        out = (ctypes.c_int * 5)()
        lib.plan(*args, out)
        return dict(zip(("apart", "waves", "columns", "blocks", "parts"), out))
    return ask


def kernel_of(got):
    return "shared" if not got["apart"] else f"{got['waves']} waves"


# steps of the loop that a piece of so many tiles has: two tiles a step with eight waves, every fourth tile of a wave where waves share columns
def steps_of(kernel, tiles):
    return {"shared": tiles // 4, "4 waves": tiles, "8 waves": -(-tiles // 2)}[kernel]


def piece_tiles(got, lens, m, share, chain):
    """Tiles of every piece, block by block: a block's tiles are those up to the last place that one of its columns sees; parts are equal but for the last."""
    out = []
    for block in range(got["blocks"]):
        last_row = (min((block + 1) * got["columns"], m * share) - 1) // share
        tiles = [-(-(at + (last_row + 1 if chain else m)) // 32) for at in lens]
        if not got["parts"]:
            out += tiles
            continue
        each, before = -(-sum(tiles) // got["parts"]), 0
        for mine in tiles:
            for part in range(got["parts"]):
                held = min((part + 1) * each, before + mine) - max(part * each, before)
                if held > 0:
                    out.append(held)
            before += mine
    return out


def filled(lens, m, kv_heads, d, page, dtype, seed):
    """A cache whose places, the rows' own among them, hold random keys and values, and what stands there by sequence."""
    cache = Cache([0] * len(lens), max(at + m for at in lens), kv_heads, d, page, dtype, seed=seed)          # pages for all, in any order, with NaNs
    cache.lens_list, cache.m = list(lens), m
    gen = torch.Generator().manual_seed(seed)
    held = []
    for s, at in enumerate(lens):
        places = torch.arange(at + m)
        k, v = (torch.randn(at + m, kv_heads, d, generator=gen).to(dtype) for _ in range(2))
        pages = torch.tensor(cache.table[s])[places // page]
        cache.k[pages, :, places % page] = k
        cache.v[pages, :, places % page // 8, :, places % 8] = v
        held.append((k, v))
    return cache, held


def seen_by_rows(at, m, parents):
    """[m][at + m]: which places each row sees."""
    seen = torch.zeros(m, at + m, dtype=torch.bool)
    seen[:, :at] = True
    for i in range(m):
        if parents is None:
            seen[i, at:at + i + 1] = True
        else:
            up = int(parents[i])
            if 0 <= up < i:
                seen[i] = seen[up]
            seen[i, at + i] = True
    return seen


def queries(held, seen, m, kv_heads, share, d, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    q = torch.randn(len(held), m, kv_heads * share, d, generator=gen) * 2.0
    ahead = 25.0 / (d ** 0.5 - 3.5) if d >= 40 else 12.0                 # scores of the place looked for lie about 25 over the others'
    for s, (k, _) in enumerate(held):
        for i in range(m):
            places = seen[s][i].nonzero().flatten()
            for h in range(kv_heads * share):
                x = i * share + h % share
                if (x + h // share) % 2 == 0 and len(places):
                    q[s, i, h] = ahead * k[places[(x * 61 + s * 17 + h // share * 29) % len(places)], h // share].float()
    return q.to(dtype)


def plain(q, held, seen, share):
    """-> out, lse, sums of weights times |v|, the largest sums of |q||k|, in 64 bits."""
    n, m, heads, d = q.shape
    out, size = torch.zeros((n, m, heads, d), dtype=torch.float64), torch.zeros((n, m, heads, d), dtype=torch.float64)
    lse, reach = torch.full((n, m, heads), -math.inf, dtype=torch.float64), torch.zeros((n, m, heads), dtype=torch.float64)
    for s, (k, v) in enumerate(held):
        some = seen[s].any(dim=1)
        for h in range(heads):
            x, keys, values = q[s, :, h].double(), k[:, h // share].double(), v[:, h // share].double()
            score = (x @ torch.nan_to_num(keys, nan=0.0, posinf=0.0, neginf=0.0).t() * d ** -0.5).masked_fill(~seen[s], -math.inf)
            w = torch.nan_to_num(torch.softmax(score, dim=1))
            used = seen[s].any(dim=0)                                    # places that no row sees are none of anyone's
            values = torch.where(used[:, None], values, 0.0)
            odd = ~torch.isfinite(values)
            out[s, :, h] = w @ torch.where(odd, 0.0, values)
            for p in odd.any(dim=1).nonzero().flatten().tolist():        # seldom: 0 times infinity is no number
                for i in seen[s][:, p].nonzero().flatten().tolist():
                    out[s, i, h] += torch.where(odd[p], values[p] * w[i, p], 0.0)
            size[s, :, h] = w @ torch.where(odd, 0.0, values).abs()
            lse[s, some, h] = torch.logsumexp(score[some], dim=1)
            reach[s, :, h] = ((x.abs() @ torch.nan_to_num(keys, nan=0.0, posinf=0.0, neginf=0.0).abs().t()) * seen[s]).amax(dim=1) * d ** -0.5
    return out, lse, size, reach


def compare(P, q, cache, held, seen, share, parents, max_places):
    k, v, table, lens = cache.gpu()
    got, lse = P.ivfpq_draft_attention(q.cuda(), k, v, table, lens, parents=None if parents is None else parents.cuda(), max_places=max_places, with_lse=True)
    again = P.ivfpq_draft_attention(q.cuda(), k, v, table, lens, parents=None if parents is None else parents.cuda(), max_places=max_places)
    assert torch.equal(got.view(torch.int16), again.view(torch.int16))                     # the same bits again
    want, want_lse, size, reach = plain(q, held, seen, share)
    got, lse, d, u = got.cpu().double(), lse.cpu().double(), q.shape[3], half_step(cache.dtype)
    longest = max(cache.lens_list) + cache.m
    sums = (longest + 64) * 2.0 ** -24
    scores = torch.expm1(2 * (d + 4) * 2.0 ** -24 * reach + 2.0 ** -18)[..., None]
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    cut = longest * 2.0 ** -31 * float(size.max())
    most = (u + scores + 2 * sums) * size + u * want.abs() * (1 + 2 * u) + cut + (2.0 ** -25 if cache.dtype == FP16 else 0.0)
    off = torch.where(fine, (got - want).abs(), 0.0)
    assert bool((off <= torch.where(fine, most, 0.0)).all()), (float(off.max()), float(torch.where(fine, off - most, 0.0).max()))
    some = torch.isfinite(want_lse)
    assert torch.equal(torch.isneginf(lse), torch.isneginf(want_lse))
    allowed = (d + 4) * 2.0 ** -24 * reach + 2.0 ** -18 + sums + 2.0 ** -22 * torch.where(some, want_lse, 0.0).abs()
    assert bool((torch.where(some, (lse - want_lse).abs(), 0.0) <= allowed).all())


LENS = [1_500, 703, 992, 1_311]
# kernel, m, share, kv_heads, d, page, trees
SHAPES = [("8 waves", 64, 3, 2, 128, 32, True), ("8 waves", 50, 8, 1, 64, 16, True), ("8 waves", 130, 1, 2, 128, 256, False), ("8 waves", 260, 2, 1, 80, 64, False),
          ("8 waves", 43, 6, 1, 120, 16, True), ("8 waves", 257, 1, 1, 40, 16, False),
          ("4 waves", 24, 2, 2, 128, 16, True), ("4 waves", 64, 1, 1, 64, 32, True), ("4 waves", 33, 3, 1, 256, 64, False), ("4 waves", 20, 1, 2, 256, 16, True),
          ("4 waves", 100, 1, 1, 80, 256, False), ("4 waves", 17, 2, 1, 136, 32, False),
          ("shared", 1, 4, 4, 128, 16, False), ("shared", 1, 20, 2, 64, 32, False), ("shared", 8, 4, 2, 128, 256, True), ("shared", 16, 1, 2, 256, 64, True),
          ("shared", 1, 1, 3, 40, 16, False), ("shared", 11, 2, 1, 80, 32, False)]


def prepare(shape, dtype, lens):
    _, m, share, kv_heads, d, page, trees = shape
    parents = tree(len(lens), m, m) if trees else None
    cache, held = filled(lens, m, kv_heads, d, page, dtype, seed=m + d)
    seen = [seen_by_rows(at, m, None if parents is None else parents[s]) for s, at in enumerate(lens)]
    return cache, held, seen, parents


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda x: "-".join(map(str, x)))
def test_whole_sequences(P, plan, shape, dtype):
    """Pieces that are whole sequences, with odd and even numbers of tiles."""
    kernel, m, share, kv_heads, d, page, trees = shape
    got = plan(len(LENS), m, kv_heads * share, kv_heads, d, 0)
    tiles = piece_tiles(got, LENS, m, share, not trees)
    assert kernel_of(got) == kernel and not got["parts"] and min(steps_of(kernel, t) for t in tiles) >= (5 if kernel == "shared" else 10) and {t % 2 for t in tiles} == {0, 1}
    cache, held, seen, parents = prepare(shape, dtype, LENS)
    compare(P, queries(held, seen, m, kv_heads, share, d, dtype, m), cache, held, seen, share, parents, 0)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("lens", [[1_900], [1_500, 703, 992]])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda x: "-".join(map(str, x)))
def test_divided_sequences(P, plan, shape, lens, dtype):
    """Long pieces of one sequence alone, and of several whose parts end inside of sequences: max_places, which only divides, asks for few parts."""
    kernel, m, share, kv_heads, d, page, trees = shape
    n, wanted = len(lens), 3 if len(lens) == 1 else 5
    bound = -(-wanted * (128 if kernel != "shared" else 256) // n)
    got = plan(n, m, kv_heads * share, kv_heads, d, bound)
    tiles = piece_tiles(got, lens, m, share, not trees)
    assert kernel_of(got) == kernel and got["parts"] == wanted and len(tiles) > n * got["blocks"]
    assert max(steps_of(kernel, t) for t in tiles) >= (5 if kernel == "shared" else 10)
    cache, held, seen, parents = prepare(shape, dtype, lens)
    compare(P, queries(held, seen, m, kv_heads, share, d, dtype, m), cache, held, seen, share, parents, bound)


@pytest.mark.parametrize("parts", [0, 3])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda x: "-".join(map(str, x)))
def test_pages_that_are_missing_late(P, plan, shape, parts):
    """A page that is not there two thirds on, so that the rest of the piece goes with masks, and a second one near the end; infinities and NaNs in a row that few see."""
    kernel, m, share, kv_heads, d, page, trees = shape
    lens, dtype = [1_911, 1_650], BF16
    bound = -(-parts * (128 if kernel != "shared" else 256) // len(lens))
    got = plan(len(lens), m, kv_heads * share, kv_heads, d, bound)
    assert kernel_of(got) == kernel and got["parts"] == parts
    cache, held, seen, parents = prepare(shape, dtype, lens)
    for s, at in enumerate(lens):
        for missing in (at * 2 // 3 // page, (at - 1) // page - 1):
            cache.table[s][missing] = -1 - s
            seen[s][:, missing * page:(missing + 1) * page] = False
        if m > 2:
            k, v = held[s]
            place = at + m - 2
            v[place, :, 1::3] = (math.inf, math.nan)[s]
            cache.v[cache.table[s][place // page], :, place % page // 8, :, place % 8] = v[place]
    compare(P, queries(held, seen, m, kv_heads, share, d, dtype, m), cache, held, seen, share, parents, bound)
