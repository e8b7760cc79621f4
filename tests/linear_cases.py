"""Sizes for which bpe_linear takes each of its tiles: (tile, whether k is cut into parts, m, n, k)."""
CASES = [
    # edges in every direction, a last block that is cut off
    (0, False, 33, 65, 243), (1, False, 55, 18425, 169), (2, False, 173, 7845, 291), (3, False, 131, 33249, 942), (4, False, 779, 3929, 327), (5, False, 946, 12821, 323),
    (0, True, 38, 66, 718), (1, True, 5, 28741, 2338), (2, True, 1706, 66, 2377), (3, True, 173, 8307, 7746), (4, True, 1552, 142, 3869), (5, True, 610, 3315, 4342),
    # whole tiles, whole blocks
    (0, False, 32, 128, 64), (1, False, 32, 13824, 64), (2, False, 192, 6912, 320), (3, False, 320, 11776, 1920), (4, False, 512, 5888, 384), (5, False, 1280, 9984, 384),
    (0, True, 32, 128, 768), (2, True, 128, 2816, 1472), (4, True, 128, 4480, 2752), (5, True, 768, 2816, 4544),
    # one block and two
    (0, False, 19, 66, 31), (1, False, 17, 19070, 60), (2, False, 65, 49422, 115), (4, False, 194, 32341, 114),
    # a batch of tokens over a large vocabulary
    (3, False, 64, 100256, 4096),
]
