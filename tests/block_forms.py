"""Sizes of products with step sizes per block of 128, each with the form that is meant to take it: (batch, M, N, K, edge of the tile, parts of K, workgroups).  The
form is chosen by reckoned times, whose constants may be fitted anew; test_block_forms.py holds these sizes to their forms, test_gpu_blocks.py runs them."""

# 256: workgroups (at most 256) that go from tile to tile, and more tiles than that
LARGE = [
    (1, 4000, 8000, 400, 256, 1, 512),             # rows that end within a slab, tiles that hang over
    (1, 4000, 8000, 144, 256, 1, 512),             # two slabs, the last one of 16 bytes
    (1, 4096, 8192, 128, 256, 1, 512),             # one whole slab a tile
    (1, 3828, 4383, 16, 256, 1, 270),              # 16 bytes a tile, rows of odd length
    (1, 8192, 4096, 1024, 256, 1, 512),
    (384, 512, 512, 64, 256, 1, 1536),             # attention scores
    (384, 512, 500, 48, 256, 1, 1536),
    (5, 2000, 4100, 272, 256, 1, 680),
]
# 256, the contraction in parts
LARGE_SPLIT = [
    (1, 4096, 1024, 16384, 256, 4, 256),           # weight gradients
    (2, 2048, 1024, 16384, 256, 4, 256),
    (1, 1101, 3761, 3952, 256, 2, 150),            # parts of 15 and 16 slabs
    (1, 212, 8295, 3872, 256, 4, 132),
    (2, 4299, 219, 4336, 256, 4, 136),
    (1, 143, 5517, 6368, 256, 8, 176),
    (1, 758, 708, 9584, 256, 16, 144),
    (3, 807, 4079, 16320, 256, 4, 768),            # in parts, several a workgroup
    (3, 685, 7325, 15744, 256, 4, 1044),
]
MIDDLE = [
    (1, 600, 7549, 512, 128, 1, 295),
    (2, 294, 8604, 512, 128, 1, 408),
    (5, 1365, 4669, 16, 128, 1, 2035),
    (1, 2048, 2048, 2048, 128, 1, 256),
]
MIDDLE_SPLIT = [
    (1, 1024, 1024, 16384, 128, 8, 512),           # a weight gradient
    (1, 66, 2156, 5664, 128, 8, 136),              # parts of five and six slabs
    (1, 342, 5968, 6032, 128, 2, 282),
    (2, 69, 8890, 5248, 128, 2, 280),
    (5, 66, 952, 6736, 128, 4, 160),
    (1, 65, 1110, 11952, 128, 16, 144),
]
SMALL = [
    (1, 1300, 1300, 4096, 64, 1, 441),
    (3, 700, 900, 4000, 64, 1, 495),
    (3, 2, 1537, 8112, 64, 16, 1200),
    (5, 1, 587, 4160, 64, 4, 200),
    (1, 60, 131, 2304, 64, 4, 12),
]
# few tokens: more slabs than a wavefront has ahead at the start
FEW = [
    (3, 1, 1360, 4224, 0, 1, 255),
    (5, 3, 1608, 8032, 0, 1, 505),
    (5, 22, 816, 3408, 0, 1, 255),
    (2, 53, 305, 704, 0, 1, 40),
]
FORMS = LARGE + LARGE_SPLIT + MIDDLE + MIDDLE_SPLIT + SMALL + FEW
