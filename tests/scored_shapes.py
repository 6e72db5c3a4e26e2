"""Calls of attention with masked and reshaped scores that the tests on the GPU make, with the kernel that each is there for: which one a call gets is a
matter of prices, so the tests of plans on the host hold every line."""
from collections import namedtuple

# t, H, Hkv, dh: the context's.  pages: over pages.  lists: with a row list (else all tokens).  lengths: with a length for every sequence.  B sequences of L
# keys at most, cap rows; the context has room for B sequences of `room` tokens (over pages one).  Then what is planned: rows of a tile, whether keys are
# split, who merges the splits ("last": the workgroup that comes last, "launch"), whether copies go past the L2.
Shape = namedtuple("Shape", "t H Hkv dh pages lists lengths B L cap room bq split merge once")


def dense(t, H, Hkv, dh, B, L, cap, bq, merge="", once=False, lengths=False, lists=True, room=0):
    return Shape(t, H, Hkv, dh, False, lists, lengths, B, L, cap, room or L, bq, merge != "", merge, once)


def paged(t, H, Hkv, dh, B, L, cap, bq, merge="", once=False, room=4096):
    return Shape(t, H, Hkv, dh, True, True, True, B, L, cap, room, bq, merge != "", merge, once)


# Splits of every kind, of up to 64 sequences and of more (test_gpu_scored_offsets.py)
SPLITS = [
    dense("f32", 4, 2, 64, 3, 3000, 12, 2, "last"), dense("f32", 4, 2, 64, 70, 1000, 210, 32, "last"), dense("bf16", 4, 2, 64, 3, 3000, 12, 32, "last"),
    dense("bf16", 4, 4, 128, 3, 2000, 36, 128, "launch"), dense("bf16", 8, 2, 128, 70, 1000, 210, 128, "launch", True, lengths=True),
    dense("bf16", 4, 2, 64, 70, 1000, 210, 128, "last", True), paged("bf16", 4, 2, 64, 3, 3008, 12, 32, "last"), paged("f32", 4, 2, 64, 3, 3008, 12, 2, "last"),
]

# Caps in fp32 (test_gpu_scored_caps.py)
CAPS = [dense("f32", 8, 2, 64, 1, 200, 3, 2), dense("f32", 4, 4, 128, 1, 200, 5, 2, "last"), dense("f32", 8, 2, 64, 1, 500, 500, 32), dense("f32", 8, 8, 128, 1, 500, 400, 32)]

# The 128-row kernel of bf16 over [B, L] caches: one group of heads a tile and several, heads of 64 and 128, past the L2, all tokens, key splits of either
# merge (test_gpu_scored_kernels.py, which gives the rows of each sequence).
MANY = [dense("bf16", 16, 16, 128, 2, 500, 800, 128), dense("bf16", 28, 4, 128, 2, 300, 461, 128), dense("bf16", 32, 32, 64, 2, 500, 800, 128),
        dense("bf16", 16, 2, 64, 2, 700, 1200, 128), dense("bf16", 32, 32, 64, 16, 300, 1920, 128, once=True)]
MANY_LENGTHS = [dense("bf16", 16, 16, 128, 2, 500, 800, 128, lengths=True), dense("bf16", 16, 2, 64, 2, 700, 1200, 128, lengths=True),
                dense("bf16", 32, 32, 64, 16, 300, 1920, 128, once=True, lengths=True)]
MANY_ALL = [dense("bf16", 16, 16, 128, 2, 400, 800, 128, lists=False), dense("bf16", 32, 8, 64, 2, 600, 1200, 128, lists=False)]
MANY_SPLIT = [dense("bf16", 4, 4, 128, 3, 2000, 36, 128, "launch"), dense("bf16", 4, 2, 64, 70, 1000, 210, 128, "last", True)]
# ... and over pages
MANY_PAGES = [paged("bf16", 16, 16, 128, 3, 512, 800, 128), paged("bf16", 28, 4, 128, 3, 512, 500, 128), paged("bf16", 16, 2, 64, 3, 704, 1200, 128),
              paged("bf16", 32, 32, 128, 8, 320, 600, 128, once=True)]
# The 32-row kernel of fp32
TILE = [dense("f32", 8, 2, 64, 1, 500, 500, 32, room=4096), dense("f32", 8, 8, 128, 2, 300, 461, 32), dense("f32", 8, 2, 128, 2, 300, 461, 32)]
TILE_LENGTHS = [dense("f32", 8, 8, 128, 2, 300, 461, 32, lengths=True)]
TILE_ALL = [dense("f32", 8, 8, 128, 2, 150, 300, 32, lists=False)]
TILE_SPLIT = [dense("f32", 4, 2, 64, 2, 3000, 200, 32, "last"), dense("f32", 4, 2, 64, 70, 1000, 210, 32, "last")]
TILE_PAGES = [paged("f32", 8, 2, 64, 4, 384, 460, 32), paged("f32", 8, 8, 128, 4, 384, 460, 32), paged("f32", 4, 4, 128, 3, 2048, 60, 32, "last")]
# Values that are no numbers, in both
NO_NUMBER = [dense("bf16", 16, 16, 128, 1, 1000, 700, 128, room=4096), dense("bf16", 32, 4, 64, 1, 1000, 800, 128, room=4096),
             dense("f32", 8, 8, 128, 1, 200, 150, 32, room=4096), dense("f32", 8, 8, 64, 1, 200, 150, 32, room=4096)]
# Scores without a bound, in each of the four kernels (test_gpu_scored_infinite.py)
INFINITE = [dense("bf16", 4, 2, 64, 1, 200, 20, 32, room=4096), dense("bf16", 16, 16, 128, 1, 1000, 700, 128, room=4096), dense("f32", 8, 2, 64, 1, 200, 3, 2),
            dense("f32", 8, 8, 128, 1, 200, 150, 32, room=4096)]
ALL = (SPLITS + CAPS + MANY + MANY_LENGTHS + MANY_ALL + MANY_SPLIT + MANY_PAGES + TILE + TILE_LENGTHS + TILE_ALL + TILE_SPLIT + TILE_PAGES + NO_NUMBER + INFINITE)
