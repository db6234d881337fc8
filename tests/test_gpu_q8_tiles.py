"""The kernels of tiles of the 8-bit product, at sizes that take them: sums are whole numbers, so everything is compared exactly, with
64-bit products of whole numbers below 2^53 scaled in the stated order in fp32 and rounded once."""
import pytest
import torch

from util_products import FAR, LAYOUTS, TILES

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


def codes_of(n, k, seed, extra=0):
    """Codes over the whole range with other bytes between the rows."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    room = torch.randint(-128, 128, (n, -(-k // 16) * 16 + extra), generator=gen, dtype=torch.int8, device="cuda")
    return room[:, :k], torch.rand(n, generator=gen, device="cuda") + 0.1


def product(a, sa, b, sb, bias, dtype):
    sums = a.double() @ b.double().t().contiguous()
    out = (sa[:, None] * sb[None, :]) * sums.float()
    return (out if bias is None else out + bias).to(dtype)


@pytest.mark.parametrize("m,n,k,tile,aligned", TILES)
def test_products(P, m, n, k, tile, aligned):
    a, sa = codes_of(m, k, seed=m, extra=16 * (m % 3))
    b, sb = codes_of(n, k, seed=n + 1, extra=16 * (n % 2))
    bias = torch.randn(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(k))
    for dtype in DTYPES:
        for with_bias in (None, bias):
            out = P.ivfpq_q8_matmul(a, sa, b, sb, bias=with_bias, out_dtype=dtype)
            assert torch.equal(out, product(a, sa, b, sb, with_bias, dtype)), dtype


@pytest.mark.parametrize("m,n,k,tile", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_layouts(P, m, n, k, tile, dtype):
    a, sa = codes_of(m, k, seed=1)
    b, sb = codes_of(n, k, seed=2, extra=32)
    want = product(a, sa, b, sb, None, dtype)
    # between guards, in rows that begin anywhere and in rows that begin at multiples of 64 bytes
    for left, right in ((3, 6), (32, -n % 32 + 32)):
        wide = torch.full((m, n + left + right), 7.0, dtype=dtype, device="cuda")
        out = P.ivfpq_q8_matmul(a, sa, b, sb, out=wide[:, left:n + left])
        assert torch.equal(out, want) and (wide[:, :left] == 7).all() and (wide[:, n + left:] == 7).all()
    # rows that are not 16 bytes apart, whose last one ends with its tensor, or every other one
    assert torch.equal(P.ivfpq_q8_matmul(a.contiguous(), sa, b.contiguous(), sb, out_dtype=dtype), want)
    stride = -(-k // 16) * 16 + 16
    tight = torch.empty(stride * (n - 1) + k, dtype=torch.int8, device="cuda").as_strided((n, k), (stride, 1))
    tight.copy_(b)
    assert torch.equal(P.ivfpq_q8_matmul(a, sa, tight, sb, out_dtype=dtype), want)
    twice = torch.stack([b, torch.zeros_like(b)], dim=1).reshape(2 * n, k)
    padded = torch.zeros((2 * n, stride), dtype=torch.int8, device="cuda")
    padded[:, :k] = twice
    assert torch.equal(P.ivfpq_q8_matmul(a, sa, padded[::2, :k], sb, out_dtype=dtype), want)


@pytest.mark.parametrize("far,m,n,k,tile", FAR)
def test_rows_far_apart(P, far, m, n, k, tile):
    """Rows 2^24 bytes apart: the last of a tile's begins up to 255 * 2^24 bytes from its first."""
    stride = 1 << 24
    a, sa = codes_of(m, k, seed=3)
    b, sb = codes_of(n, k, seed=4)
    near, rows = (a, m) if far == "a" else (b, n)
    room = torch.zeros(stride * (rows - 1) + -(-k // 16) * 16, dtype=torch.int8, device="cuda").as_strided((rows, k), (stride, 1))
    room.copy_(near)
    got = P.ivfpq_q8_matmul(room, sa, b, sb) if far == "a" else P.ivfpq_q8_matmul(a, sa, room, sb)
    assert torch.equal(got, product(a, sa, b, sb, None, torch.float32))


def test_the_same_bits_again(P):
    """Many slices, loaded while others are multiplied: the same sums every time."""
    m, n, k = 2048, 8192, 4096
    a, sa = codes_of(m, k, seed=5)
    b, sb = codes_of(n, k, seed=6)
    first = P.ivfpq_q8_matmul(a, sa, b, sb, out_dtype=torch.bfloat16)
    for _ in range(20):
        assert torch.equal(P.ivfpq_q8_matmul(a, sa, b, sb, out_dtype=torch.bfloat16), first)
