"""Sizes at which the operators in eight bits take each form of their tiles, whole and ragged: what the GPU tests run and what the launches of these sizes are checked to be."""

# M, N, K of a product -> form of its tiles (256 x 256, 128 x 128, 128 x 64), whether the contraction is split
PRODUCTS = {
    (4096, 4096, 128): ("wide", False),          # whole tiles of one K-tile
    (3900, 4090, 900): ("wide", False),          # ragged on every side, rows of the result on 4 bytes in either type
    (8190, 4095, 200): ("wide", False),          # two tiles a block, rows on 2 bytes
    (2048, 2048, 40960): ("wide", True),
    (1990, 2041, 40000): ("wide", True),
    (3000, 760, 40000): ("wide", True),          # the shape of a weight gradient
    (2048, 2048, 640): ("square", False),
    (2000, 1999, 520): ("square", False),
    (2900, 2999, 130): ("square", False),        # three tiles a block
    (700, 500, 20000): ("square", True),
    (200, 300, 700): ("thin", False),
    (300, 401, 9000): ("thin", True),
}

# ... of which every pair of formats is run, in both types of result
ALL_FORMATS = [(3900, 4090, 900), (2000, 1999, 520), (200, 300, 700)]

# T, V, D of a training step, type -> forms of the gradient of the logits, of d_h and of d_w; pieces of the vocabulary; whether the contraction of d_h is split
LOSSES = {
    (4000, 35001, 2000, "bfloat16"): ("wide", "wide", "wide", 2, True),
    (4096, 9000, 2048, "bfloat16"): ("wide", "wide", "wide", 1, True),          # operands as they are, whole tokens and widths
    (4100, 9001, 2040, "bfloat16"): ("wide", "wide", "wide", 1, False),
    (4000, 13001, 2000, "float32"): ("wide", "wide", "wide", 2, True),
    (300, 11001, 776, "bfloat16"): ("square", "square", "wide", 1, True),
    (300, 11001, 776, "float32"): ("square", "square", "wide", 1, True),
}
