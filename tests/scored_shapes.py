"""Calls of attention with masked and reshaped scores that the tests on the GPU make, with the kernel that each is there for: which one a call gets is a
matter of prices, so the tests of plans on the host hold every line."""
from collections import namedtuple

# t, H, Hkv, dh: the context's.  pages: over pages.  lists: with a row list (else all tokens).  lengths: with a length for every sequence.  B sequences of L
# keys at most, cap rows; the context has room for B sequences of `room` tokens (over pages one).  Then what is planned: rows of a tile, whether keys are
# split, who merges the splits ("last": the workgroup that comes last, "launch"), whether copies go past the L2.
Shape = namedtuple("Shape", "t H Hkv dh pages lists lengths B L cap room bq split merge once")


def dense(t, H, Hkv, dh, B, L, cap, bq, merge="", once=False, lengths=False, lists=True):
    return Shape(t, H, Hkv, dh, False, lists, lengths, B, L, cap, L, bq, merge != "", merge, once)


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
