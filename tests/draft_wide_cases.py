"""Trees in wide tiles, by the rules of a partition of 8 CUs: (tokens before, rows, key heads, query heads, window, whether a tile is cut).  All are of heads
of 64 in either type, and of 128 in bf16."""
CUS = 8
WIDE = [("bf16", 64), ("fp32", 64), ("bf16", 128)]
CASES = {
    "whole": ([70], [90], 2, 16, 0, False),                                     # the last of six tiles has 80 of 128 columns
    "whole under a window": ([300], [90], 2, 16, 64, False),
    "several": ([130, 40, 0], [64, 33, 70], 2, 16, 0, False),
    "cut": ([2600, 20, 0], [10, 40, 35], 2, 16, 0, True),                       # one sequence of three is long
    "cut under a window": ([2600, 20, 0], [10, 40, 35], 2, 16, 1100, True),
    "cut, two tiles": ([40, 0, 2600, 70], [40, 3, 30, 12], 2, 16, 0, True),
    "cut in twelve": ([12000, 5], [5, 80], 1, 16, 0, True),
}
# ... and on 256 CUs, in narrow tiles that are cut
NARROW = {
    "one": ([3000], [13], 2, 8, 0, True),
    "two, of which one is short": ([5000, 10], [20, 3], 1, 4, 0, True),
    "under a window": ([5000, 10], [20, 3], 1, 4, 2600, True),
}
