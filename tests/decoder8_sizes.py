"""Sizes of the 8-bit decoder operators that take each of their kernels, with
work for it: remainders in rows, outputs and k, more stages of k than a kernel
holds, and whole ones.  The host tests ask the library that each still takes its
kernel, and that no kernel is without a size; the GPU tests run them."""

# outputs x rows of a workgroup: the kernel's template arguments
TILES = {
    "256x256": "Tile<4, 2, 2, 4, 1, 128, 2>",
    "128x256": "Tile<2, 2, 2, 4, 1, 64, 3>",
    "128x128": "Tile<2, 1, 2, 4, 1, 128, 4>",
    "128x128 pair": "Tile<2, 1, 2, 4, 1, 128, 2>",
    "64x128": "Tile<1, 1, 2, 4, 1, 128, 3>",
    "64x64": "Tile<1, 1, 2, 2, 1, 128, 3>",
    "32x32": "Tile<1, 1, 1, 1, 8, 256, 4>",
    "64x128 shared": "Tile<1, 1, 2, 4, 2, 256, 3>",
    "64x64 shared": "Tile<1, 1, 2, 2, 2, 256, 3>",
    "64x32 shared": "Tile<1, 1, 2, 1, 4, 256, 4>",
}

# kernel, second launch -> (m, n, k)
MATMUL = {
    ("rows 16", None): [(1, 34, 12112), (4, 1, 9984), (41, 27, 4096), (110, 478, 5696)],
    ("rows 16 few", None): [(1, 35, 944), (11, 1, 640), (23, 341, 80), (47, 571, 1648), (113, 399, 192), (191, 69, 208)],
    ("rows 32", None): [(1, 16147, 1088), (2, 28536, 640), (8, 15070, 112), (31, 16340, 16)],
    ("32x32", None): [(19, 58, 5648), (15, 114, 6656), (74, 1325, 2352), (331, 1, 64)],
    ("32x32", "join"): [(9, 40, 13200), (32, 4, 8192)],
    ("64x64", None): [(319, 919, 528), (55, 6089, 512), (395, 1, 16)],
    ("64x128", None): [(1214, 1011, 544), (325, 3020, 512), (86, 8598, 16), (2048, 1024, 1024)],
    ("128x128", None): [(150, 11124, 1488), (2574, 1479, 1792), (101, 21730, 2032)],
    ("128x128 pair", None): [(65, 17788, 432), (433, 8841, 384), (84, 16798, 16)],
    ("128x256", None): [(1317, 10326, 288), (2367, 17525, 256), (672, 12367, 16)],
    ("256x256", None): [(516, 14565, 1968), (6251, 1471, 2048)],
    ("256x256", "tail"): [(203, 18099, 9488), (5778, 751, 9728)],
    ("64x128 shared", None): [(334, 2926, 2096), (1405, 1048, 2304)],
    ("64x128 shared", "join"): [(698, 326, 16000), (688, 394, 12800)],
    ("64x64 shared", None): [(65, 6783, 1488), (107, 6626, 4608)],
    ("64x64 shared", "join"): [(43, 2538, 14576), (2154, 38, 11984)],
    ("64x32 shared", None): [(2, 13028, 3872), (53, 5883, 1280), (3863, 67, 752)],
    ("64x32 shared", "join"): [(65, 730, 13296), (1819, 63, 9728)],
}
# rows of x that lie `apart` bytes from each other: (m, n, k, apart)
MATMUL_FAR = [(150, 6001, 1040, 1 << 27), (33, 300, 8192, 1 << 28)]
# the same with the last offsets between 2^31 and 2^32
MATMUL_NEAR = [(33, 300, 8192, 1 << 27), (140, 6001, 1040, 1 << 25)]

# kernel, second launch; "few": workgroups for as many experts as there are routes -> (tokens, experts, top, n, k)
EXPERTS = {
    ("rows 16", None): [(8, 1, 1, 77, 7664), (18, 3, 2, 97, 4096)],
    ("rows 16 few", None): [(2, 3, 2, 36, 1104), (137, 128, 1, 1, 2048), (66, 60, 6, 99, 272)],
    ("rows 32", None): [(5, 32, 7, 388, 1472), (2, 8, 4, 1856, 1152), (47, 64, 4, 7887, 608)],
    ("rows 16", "few"): [(3, 128, 7, 90, 8032), (16, 1024, 5, 10, 4096)],
    ("rows 16 few", "few"): [(3, 256, 8, 40, 1104), (1, 32, 1, 548, 640)],
    ("rows 32", "few"): [(14, 60, 2, 1087, 656), (5, 64, 2, 1507, 896)],
    ("32x32", None): [(25, 3, 2, 48, 1328), (57, 4, 3, 5, 1536)],
    ("64x64", None): [(785, 16, 2, 142, 656), (2208, 16, 7, 1, 512)],
    ("64x128", None): [(530, 1, 1, 1885, 624), (2933, 8, 6, 17, 512), (3308, 32, 8, 36, 576)],
    ("128x128", None): [(406, 16, 3, 1756, 1200), (632, 64, 7, 321, 1920), (326, 8, 4, 1353, 3872)],
    ("128x128 pair", None): [(171, 70, 6, 739, 592), (321, 32, 5, 1382, 384)],
    ("128x256", None): [(966, 32, 7, 946, 608), (2327, 4, 3, 1959, 256)],
    ("256x256", None): [(1183, 5, 4, 1672, 1824), (2794, 2, 2, 4416, 1536)],
    ("256x256", "tail"): [(4312, 3, 2, 936, 4848), (4857, 64, 8, 235, 6272)],
    ("64x128 shared", None): [(236, 8, 6, 481, 2640), (3400, 16, 7, 18, 1792)],
    ("64x64 shared", None): [(622, 8, 6, 130, 1104), (1613, 16, 6, 34, 1760)],
    ("64x32 shared", None): [(11, 128, 8, 98, 7024), (229, 8, 8, 131, 1792)],
}
# (tokens, experts, top, n, k, apart)
EXPERTS_FAR = [(70, 3, 2, 131, 1040, 1 << 26), (300, 2, 1, 70, 640, 1 << 24)]
EXPERTS_NEAR = [(62, 3, 2, 131, 1040, 1 << 26), (250, 2, 1, 70, 640, 1 << 24)]

# launches with an order -> (tokens, experts, top)
ROUTE = {
    ("route_experts_kernel",): [(32, 64, 4), (16, 128, 8), (8, 256, 8), (8, 512, 3), (4, 1024, 32)],
    ("route_experts_kernel", "route_place_kernel<4>"): [(200, 64, 4), (100, 128, 8), (70, 250, 8), (60, 500, 2), (30, 1000, 9)],
    ("route_experts_kernel", "route_sum_kernel", "route_place_kernel<4>"): [(700, 60, 6), (900, 100, 2), (300, 256, 8), (300, 512, 32),
                                                                            (200, 1024, 5)],
    ("route_experts_kernel", "route_sum_kernel", "route_place_kernel<16>"): [(5000, 64, 20), (4500, 70, 32), (8200, 200, 17)],
}


ROWS = {"rows 16": "1, 16, ", "rows 16 few": "1, 8, ", "rows 32": "2, 4, "}


def name_of(kernel):
    """The name above of a kernel of the library."""
    for name, part in TILES.items() if "Tile<" in kernel else ROWS.items():
        if part in kernel:
            return name
