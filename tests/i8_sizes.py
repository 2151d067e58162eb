"""Sizes of products of 8-bit integers, rows x outputs x k, by the way they go: the kernel of few rows by its tiles of 16 rows and of 16 outputs, the others
by their tile, each with all of k or with parts of it.  test_i8_plan.py holds them to the plan, test_gpu_i8_tiles.py computes them."""

WAYS = {  # (tile, tiles of 16 rows, of 16 outputs, whether k is shared)
    ("few", 1, 1, False): [(1, 131, 272), (16, 67, 2064)],
    ("few", 1, 1, True): [(3, 35, 20016), (16, 77, 12304)],
    ("few", 1, 2, False): [(5, 4101, 400)],
    ("few", 1, 4, False): [(16, 12803, 272)],
    ("few", 2, 1, False): [(17, 131, 272), (32, 515, 1040)],
    ("few", 2, 1, True): [(17, 70, 12176), (31, 45, 40016)],
    ("few", 2, 2, False): [(30, 4101, 144)],
    ("few", 2, 4, False): [(32, 12803, 400)],
    ("few", 2, 4, True): [(19, 2051, 8208)],
    ("64 x 128", 0, 0, False): [(33, 131, 272), (129, 1031, 656)],
    ("64 x 128", 0, 0, True): [(35, 73, 1936), (100, 1001, 6416)],
    ("128 x 128", 0, 0, False): [(65, 17009, 272), (190, 12901, 1040)],
    ("128 x 128", 0, 0, True): [(591, 129, 6544), (69, 17823, 9040), (333, 5120, 13824)],
    ("192 x 256", 0, 0, False): [(259, 22235, 272), (380, 32001, 144)],
    ("192 x 256", 0, 0, True): [(138, 11205, 3808), (135, 17295, 5920)],
    ("256 x 256", 0, 0, False): [(405, 21889, 272), (1537, 8193, 400)],
    ("256 x 256", 0, 0, True): [(393, 5429, 6352), (251, 17842, 7040)],
}
ALL = [(way, size) for way, sizes in WAYS.items() for size in sizes]


def name(way):
    tile, rows, outs, shared = way
    return (tile if not rows else "%s, %d by %d" % (tile, rows, outs)) + (", k shared" if shared else "")
