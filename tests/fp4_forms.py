"""Sizes of products in 4 bits and the form that runs them, for the tests that are about one form: test_host_fp4_forms.py holds them to what the library launches, on a
runtime that runs nothing, and test_gpu_fp4_forms.py runs them."""

# name: rows, weights' rows, length, groups
SIZES = {
    "256x256": dict(m=4100, n=4110, k=1200, groups=1),
    "128x256": dict(m=2050, n=2100, k=1200, groups=1),
    "128x128": dict(m=1100, n=1030, k=1200, groups=1),
    "64x64": dict(m=16500, n=60, k=1200, groups=1),
    "thin 4 4": dict(m=200, n=4000, k=1200, groups=1),
    "thin 4 2": dict(m=100, n=1030, k=1200, groups=1),
    "thin 4 1": dict(m=60, n=1030, k=1200, groups=1),
    "thin 3 1": dict(m=40, n=1030, k=1200, groups=1),
    "thin 2 1": dict(m=30, n=1030, k=1200, groups=1),
    "thin 1 1": dict(m=7, n=1030, k=1200, groups=1),
    "thin 2 4": dict(m=100, n=300, k=1200, groups=4),
    "thin 1 2": dict(m=60, n=300, k=1200, groups=4),
}
LARGE = ["256x256", "128x256", "128x128"]

# lengths that end inside a sixteen of bytes, a block of 32, a stage of 128 and a run of four stages, beyond those that go to tiles of 128 x 128
LENGTHS = [1025, 1026, 1039, 1040, 1055, 1056, 1057, 1087, 1151, 1152, 1153, 1279, 1280, 1281, 1407, 1408, 1409, 1535, 1536, 1537, 1663, 2047, 2048, 2049]
# (form, bounds): the groups' rows
RAGGED = [("256x256", [0, 4100, 4100]), ("256x256", [0, 5, 5, 1140, 3300, 4100]), ("256x256", [3, 300, 2900, 4095]), ("256x256", [0] + [600 + 37 * g for g in range(12)] + [4100]),
          ("256x256", [0, 0, 0, 4100]), ("256x256", [0, 256, 512, 768, 1024, 4096, 4100]),
          ("128x256", [0, 2050, 2050]), ("128x256", [0, 5, 5, 700, 1500, 2050]), ("128x256", [3, 300, 1400, 2047]), ("128x256", [0, 0, 0, 2050]),
          ("128x256", [0, 128, 256, 384, 512, 2048, 2050]), ("128x256", [0] + [100 + 37 * g for g in range(12)] + [2050])]

# bounds that fall or lie outside [0, m], and what they count as
BOUNDS = {"256x256": (4000, [-5, 1000, 20, 2500, 100000], [(0, 1000), (1000, 1000), (1000, 2500), (2500, 4000)]),
          "128x256": (2040, [-5, 700, 20, 1500, 100000], [(0, 700), (700, 700), (700, 1500), (1500, 2040)]),
          "128x128": (1040, [-5, 300, 20, 700, 100000], [(0, 300), (300, 300), (300, 700), (700, 1040)])}

# weights of so many groups that the last one's values lie beyond 2^32 bytes; all rows are the last group's
FAR_WEIGHTS = {"256x256": dict(m=13500, n=8192, k=16384, groups=70), "128x256": dict(m=2400, n=8192, k=16384, groups=70), "128x128": dict(m=19300, n=16384, k=1024, groups=600),
               "thin 1 2": dict(m=600, n=8192, k=16384, groups=70), "thin 2 4": dict(m=1700, n=8192, k=16384, groups=70)}
# rows that lie so far apart that the last tiles' begin beyond 2^32 bytes
FAR_ROWS = {"256x256": 1100000 + 16, "128x256": 2100224, "128x128": (1 << 22) - 16}

# (form, rows, weights' rows, split) of the weights' gradient: dw is n x k of the groups' rows
GRADIENT = [("cols 256x256", 4100, 4110, [0, 1200, 2500]), ("cols 256x256", 2100, 2050, [0, 1, 130, 131, 1400, 1400, 3300, 4700, 6100, 9000, 13000]),
            ("cols 128x256", 2100, 2050, [0, 1300]), ("cols 128x256", 2100, 2050, [0, 1, 2300]),
            ("cols 128x128", 1030, 1100, [0, 1, 130, 131, 600, 600, 2000]), ("cols 64x64", 1100, 60, [0, 129, 300, 600, 1200, 2500])]
