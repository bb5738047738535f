"""Shapes that the library's rules send to every variant of the kernels that take many sizes, with remainders in each of them."""
from paper_1810_09868_amd import binding as B

# products of updates on 256 x 256 tiles: (batch, rows, cols)
MUON_256 = [(1, 1088, 10944), (1, 1216, 9793), (1, 9793, 1216), (4, 1270, 2500), (3, 3001, 1301)]
# 4-bit products on laid out activations: (dtype, N, In, Out) -> (tiles of 16 rows, tiles of 16 outputs)
W4_TILES = {
    (B.BF16, 16, 9500, 1000): (1, 1), (B.BF16, 16, 9500, 4111): (1, 2), (B.BF16, 15, 23999, 7777): (1, 4),
    (B.BF16, 17, 700, 77): (2, 1), (B.BF16, 31, 640, 4111): (2, 2), (B.BF16, 32, 12345, 7001): (2, 4),
    (B.BF16, 50, 1000, 130): (4, 1), (B.BF16, 100, 4096, 4096): (4, 2), (B.BF16, 130, 4095, 4503): (4, 4),
    (B.F32, 16, 4800, 1000): (1, 1), (B.F32, 9, 9001, 4111): (1, 2), (B.F32, 11, 8001, 7301): (1, 4),
    (B.F32, 17, 700, 77): (2, 1), (B.F32, 31, 640, 4111): (2, 2), (B.F32, 32, 4001, 7300): (2, 4),
    (B.F32, 50, 1000, 130): (4, 1), (B.F32, 70, 1500, 2100): (4, 2), (B.F32, 130, 2047, 2777): (4, 4),
}
