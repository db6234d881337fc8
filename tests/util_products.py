"""Sizes of 8-bit products that a test of the kernels of tiles takes, with the tile that the library's rule gives them and whether rows of
n values of 4 and of 2 bytes begin at multiples of 64 bytes."""

# m, n, k, tile, aligned (fp32, 16 bits)
TILES = [
    (300, 3001, 200, 128, (False, False)),
    (129, 3400, 16, 128, (False, False)),
    (1000, 2080, 200, 128, (True, True)),             # a slice and a part of one
    (1024, 2048, 640, 128, (True, True)),             # whole slices
    (1024, 2064, 128, 128, (True, False)),            # one whole slice
    (2600, 256, 144, 128, (True, True)),
    (4096, 4096, 1024, 256, (True, True)),
    (4100, 4224, 1000, 256, (True, True)),
    (2048, 8192, 4096, 256, (True, True)),            # many slices
    (1027, 16411, 385, 256, (False, False)),          # three slices and a byte
    (1000, 16500, 300, 256, (False, False)),
    (256, 65600, 300, 256, (True, True)),
    (65600, 256, 300, 256, (True, True)),
]
LAYOUTS = [(300, 3001, 200, 128), (1000, 16500, 300, 256)]
# rows 2^24 bytes apart: of a or of b, as many as a tile has, and as many of the other as make the library take that tile
FAR = [("b", 2600, 256, 144, 128), ("b", 65600, 256, 300, 256), ("a", 256, 65600, 300, 256)]
