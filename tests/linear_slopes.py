"""Sizes that take each kernel of the elementwise part of a linear layer's backward pass, on 256 compute units: (elements, rows ahead, rows of whole 16 bytes, n, f_out)."""
SLOPES = [
    ("16", 2, True, 1, 8), ("16", 2, True, 103, 64), ("16", 2, True, 41, 1032), ("16", 4, True, 66003, 8), ("16", 4, True, 4099, 8192), ("16", 2, False, 7, 3), ("16", 2, False, 301, 301),
    ("16", 2, False, 37, 1031), ("16", 2, False, 4099, 1001), ("16", 4, False, 66003, 13), ("16", 4, False, 70001, 5), ("16", 4, False, 35000, 1030),
    ("f32", 2, True, 1, 4), ("f32", 2, True, 103, 64), ("f32", 2, True, 41, 516), ("f32", 4, True, 66003, 8), ("f32", 4, True, 4099, 4096), ("f32", 2, False, 7, 3), ("f32", 2, False, 301, 301),
    ("f32", 2, False, 37, 1031), ("f32", 2, False, 4099, 1001), ("f32", 4, False, 66003, 13), ("f32", 4, False, 70001, 3), ("f32", 4, False, 35000, 515),
]
