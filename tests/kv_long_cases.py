"""Cases of include/kv.h's calls in which a wave takes more than one step: shared by the tests that run them and by the one that says that they do."""

# rope_qkv and its backward: B, N, Hq, Hkv, d, norm, rot, interleaved, positions given.  Heads of a token: fewer than the rows of a wave's step (8 of
# d = 128, 16 of 64), more, a multiple
ROPE = [
    (3, 5001, 1, 1, 128, True, 128, False, True), (1, 15003, 1, 1, 128, False, 128, True, False), (2, 4101, 4, 1, 128, True, 64, True, False),
    (3, 1801, 8, 1, 128, True, 128, False, False), (5, 409, 28, 4, 128, False, 96, False, True), (2, 701, 32, 8, 128, True, 128, False, False),
    (3, 1101, 12, 2, 128, True, 128, True, True), (1, 2751, 12, 2, 128, False, 128, False, False),
    (2, 15011, 1, 1, 64, True, 64, False, False), (3, 10007, 1, 1, 64, False, 48, True, True), (4, 2503, 8, 1, 64, True, 64, False, True),
    (1, 5501, 12, 2, 64, True, 32, True, False), (2, 1153, 32, 8, 64, True, 64, False, True), (3, 1201, 20, 4, 64, False, 64, False, False),
    (2, 1237, 28, 4, 64, True, 64, True, False),
]

# kv_append: T, Hq, Hkv, d, norm, rot, interleaved, page; the groups of 64 / (d / 16) heads of a token are not a multiple of four
APPEND = [
    (1103, 32, 4, 128, True, 128, False, 64), (901, 32, 8, 128, False, 64, True, 16), (2101, 9, 1, 128, True, 128, True, 32), (1501, 32, 8, 64, True, 64, False, 128),
    (2203, 14, 2, 64, False, 32, True, 16), (861, 64, 8, 64, True, 64, False, 32), (497, 56, 8, 128, True, 96, False, 256),
]
