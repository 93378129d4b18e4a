"""Products D (M x N) = A (M x K) B (K x N) that take each tile of the linear layers, with and without a split sum, on 256 compute units:
(elements, rows in whole 16 bytes, edge of the tile, in how many shares the sum is cut, M, N, K).  No size is a multiple of a tile's edge or of a stage's depth."""
PRODUCTS = [
    ("16", False, 256, 1, 3043, 3045, 139), ("16", False, 256, 42, 395, 573, 31763), ("16", False, 128, 1, 1411, 3549, 139),
    ("16", False, 128, 42, 259, 461, 18371), ("16", False, 64, 1, 75, 77, 139), ("16", False, 64, 3, 75, 77, 379),
    ("16", True, 256, 1, 3040, 3040, 139), ("16", True, 256, 28, 392, 832, 54907), ("16", True, 128, 1, 2456, 2456, 139),
    ("16", True, 128, 63, 208, 456, 45755), ("16", True, 64, 1, 72, 72, 139), ("16", True, 64, 4, 72, 72, 459),
    ("f32", False, 128, 1, 1699, 2045, 139), ("f32", False, 128, 42, 211, 261, 15307), ("f32", False, 64, 1, 75, 77, 139), ("f32", False, 64, 4, 75, 77, 211),
]
