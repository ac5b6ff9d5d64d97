"""Sizes of the 8-bit products' tests by the kernel that they are meant for: a test on the host holds them to it, so that another choice of routes
cannot leave a kernel untested.  Groups: rows of each; `behind`: rows that belong to none."""

KINDS = range(4)             # E8M0 scales, float32 scales, the same with a float32 result
FEW, TILES64, DEEP64, TILES128, TALL, BIG = range(6)

# (m, n, k).  FEW: 1 to 16, 17 to 32 and 33 to 64 rows have an instance each, with and without a cut k; large tiles: odd and even numbers of blocks
# of k, whole and not
DENSE = {
    "few rows, 16": [(1, 17, 1), (3, 130, 129), (16, 256, 512), (9, 33, 1100)],
    "few rows, 32": [(17, 40, 130), (31, 100, 777), (32, 257, 1024), (20, 19, 60)],
    "few rows, 64": [(33, 100, 777), (64, 70, 384), (50, 300, 1290)],
    "few rows, cut": [(5, 96, 20000), (25, 200, 8200), (40, 200, 16500)],
    "64 x 64, two stages": [(970, 1837, 5), (706, 1353, 145), (1900, 700, 640)],
    "64 x 64, four stages": [(65, 129, 255), (130, 257, 1000), (300, 513, 384), (257, 300, 1300)],
    "64 x 64, cut": [(75, 121, 2432), (230, 66, 2050), (126, 110, 2582)],
    "128 x 128": [(3511, 1089, 3), (1143, 2782, 139), (2600, 2500, 640)],
    "256 x 128": [(2183, 1893, 1425), (899, 4368, 1543), (1094, 3794, 1536)],
    "256 x 256": [(3867, 3169, 652), (2710, 4368, 816), (3601, 3841, 768)],
}
ROUTE = {"few rows, 16": FEW, "few rows, 32": FEW, "few rows, 64": FEW, "few rows, cut": FEW, "64 x 64, two stages": TILES64, "64 x 64, four stages": DEEP64,
         "64 x 64, cut": TILES64, "128 x 128": TILES128, "256 x 128": TALL, "256 x 256": BIG}
# kinds of operands that a route has a kernel for
HAS = {TALL: (0, 1), BIG: (0,)}

# (rows of each group, rows behind, n, k): uneven loads, empty groups, a group with most of the rows
ROWS = {
    "few rows, 16": [([300, 0, 1, 17] + [2] * 27 + [33], 3, 150, 300)],
    "few rows, 32": [([500, 0, 1, 17] + [5] * 28, 5, 270, 520)],
    "few rows, 64": [([800, 0, 65, 64] + [20] * 16, 7, 70, 700)],
    "64 x 64, two stages": [([400, 0, 1, 70, 64, 200, 100, 3, 120, 125, 130], 9, 845, 107)],
    "64 x 64, four stages": [([300, 0, 579], 4, 93, 140)],
    "128 x 128": [([1500, 1, 129, 0, 700, 383], 7, 989, 330)],
    "256 x 128": [([1, 0, 257, 1700, 256, 3, 1000, 31, 0, 100, 128, 2], 9, 961, 1436), ([500, 0, 2, 300, 100, 90, 5], 3, 2932, 1664)],
    "256 x 256": [([2000, 0, 1, 255, 700, 257, 128, 40], 6, 2948, 669), ([3000, 0, 1, 255, 1200, 257, 128, 40, 386], 0, 1960, 768)],
}
# (rows of each group, rows behind, m, n): groups of no, one, two, an odd and an even number of blocks, whole and not
CONTRACTION = {
    "64 x 64, two stages": [([100, 0, 257, 1], 6, 68, 2297)],
    "64 x 64, four stages": [([1, 0, 700], 2, 73, 142)],
    "128 x 128": [([1, 0, 128, 300, 129, 0, 40], 8, 1211, 337)],
    "256 x 128": [([1, 0, 129, 384, 6186], 5, 531, 1414)],
    "256 x 256": [([1, 0, 257, 128, 2370], 3, 1543, 1450)],
}


def columns(counts, behind):
    """Of a transpose whose groups start at whole blocks."""
    rows = sum(counts) + behind
    return (rows + 127 * min(len(counts), rows)) // 128 * 128
