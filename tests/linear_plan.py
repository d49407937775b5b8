"""Which kernel a linear layer's product goes to, asked of the built library, so that tests can say what
their sizes reach."""
import ctypes

from paper_2609_10632_amd import numbat as nb

TILES = ("256x256", "128x256", "128x128 deep", "128x128", "64x64", "64x64 any", "rows")
FWD, DATA, WEIGHT = range(3)


class _Plan(ctypes.Structure):
    _fields_ = [("tile", ctypes.c_int), ("splits", ctypes.c_int), ("k_per_split", ctypes.c_int64)]


def plan(kind, m, k, n, act=False, f32=False, ldx=0, ldy=0):
    """(tile, reduction ranges, whether a weight gradient adds up the bias gradient) for the product that
    numbat_linear_* makes of m rows, k input and n output features; act: the descriptor has an activation."""
    lib = nb.load()
    pick = lib["_ZN6numbat9gemm_pickENS_8GemmKindElilid"]
    pick.restype, pick.argtypes = _Plan, [ctypes.c_int, ctypes.c_int64, ctypes.c_int, ctypes.c_int64, ctypes.c_int,
                                          ctypes.c_double]
    sums = lib["_ZN6numbat14gemm_sums_rowsERKNS_8GemmPlanE"]
    sums.restype, sums.argtypes = ctypes.c_bool, [ctypes.POINTER(_Plan)]
    x, dy, w = (m, k, ldx or k), (m, n, ldy or n), (n, k, k)
    a, b = {FWD: (x, w), DATA: (dy, w), WEIGHT: (dy, x)}[kind]
    pack = sum(2.0 * rows * (-(-cols // 8) * 8) for rows, cols, ld in (a, b) if cols % 8 or ld % 8)
    z = 2 if act else 0
    size = {FWD: (m, n, k, (4 if f32 else 2) + z), DATA: (m, k, n, 2 + z), WEIGHT: (n, k, m, 4)}[kind]
    p = pick(kind, *size, pack)
    return TILES[p.tile], p.splits, kind == WEIGHT and bool(sums(ctypes.byref(p)))


# Sizes (m, k, n) that reach each kernel, by (tile, whether the reduction is split[, whether the weight gradient
# adds up the bias gradient on the way]).  Of each: results of whole 128-byte lines, of whole 16-byte vectors (or
# None where only odd rows go there), and odd; none a multiple of the tile, three steps or more of the reduction.
FORWARD_BF16 = {
    ("256x256", False): [(1294, 520, 8896), (19865, 392, 528), (19680, 488, 549)],
    ("256x256", True): [(550, 8016, 7104), (534, 7680, 7088), (682, 7371, 5700)],
    ("128x256", False): [(404, 648, 9024), (771, 664, 4856), (392, 1136, 9383)],
    ("128x256", True): [(147, 6632, 6208), (129, 7256, 6600), (141, 6856, 8499)],
    ("128x128 deep", False): [(129, 200, 11136), (136, 376, 10840), (203, 544, 8465)],
    ("128x128 deep", True): [(68, 4856, 4352), (77, 4960, 4272), (66, 4976, 5181)],
    ("128x128", False): [(270, 216, 11776), (286, 208, 11504), (11649, 296, 301)],
    ("128x128", True): [(132, 5392, 10880), (984, 10152, 2592), (902, 5334, 2639)],
    ("64x64", False): [(30, 200, 64), (30, 216, 136), (31, 224, 95)],
    ("64x64", True): [(30, 1824, 128), (31, 1816, 72), (31, 2088, 490)],
    ("64x64 any", False): [None, None, (32, 203, 153)],
    ("64x64 any", True): [None, None, (32, 1169, 1273)],
}
FORWARD_F32 = {
    ("256x256", False): [(8883, 888, 1344), (11010, 880, 1096), (8298, 911, 1417)],
    ("256x256", True): [(523, 8016, 7040), (664, 6936, 6040), (545, 7664, 6842)],
    ("128x256", False): [(535, 1128, 7360), (449, 1760, 8208), (761, 1336, 5415)],
    ("128x256", True): [(129, 7024, 7040), (150, 6576, 6072), (150, 7512, 6601)],
    ("128x128 deep", False): [(130, 880, 11840), (136, 1088, 11888), (131, 600, 11802)],
    ("128x128 deep", True): [(65, 4832, 4160), (65, 5080, 4592), (74, 5272, 4113)],
    ("128x128", False): [(138, 224, 8960), (129, 376, 10344), (706, 200, 2245)],
    ("128x128", True): [(902, 6424, 2688), (1312, 4984, 1832), (206, 5080, 10775)],
    ("64x64", False): [(31, 200, 128), (30, 208, 104), (30, 256, 156)],
    ("64x64", True): [(32, 1800, 64), (32, 1848, 88), (30, 2000, 358)],
    ("64x64 any", False): [None, None, (30, 204, 163)],
    ("64x64 any", True): [None, None, (31, 1243, 1193)],
}
DATA_GRADIENT = {
    ("256x256", False): [(19925, 576, 528), (19971, 528, 416), (16790, 668, 359)],
    ("256x256", True): [(517, 6656, 8240), (522, 6952, 8224), (544, 6666, 7544)],
    ("128x256", False): [(268, 11136, 912), (272, 10992, 616), (260, 11352, 931)],
    ("128x256", True): [(143, 5952, 6304), (136, 5544, 6720), (131, 8264, 5667)],
    ("128x128 deep", False): [(129, 9600, 288), (131, 9360, 216), (133, 8920, 575)],
    ("128x128 deep", True): [(66, 3136, 3512), (66, 2696, 3280), (77, 3632, 4260)],
    ("128x128", False): [(257, 11328, 544), (269, 11144, 408), (390, 9672, 401)],
    ("128x128", True): [(945, 2624, 6048), (911, 2568, 5872), (898, 2594, 5356)],
    ("64x64", False): [(32, 64, 200), (30, 136, 200), (31, 115, 267)],
    ("64x64", True): [(30, 64, 1432), (31, 136, 1464), (31, 392, 1415)],
    ("64x64 any", False): [None, None, (30, 72, 209)],
    ("64x64 any", True): [None, None, (31, 887, 1199)],
}
WEIGHT_GRADIENT = {
    ("256x256", False, False): [(4198, 3520, 3608), (4129, 3816, 3296), (4234, 3698, 3516)],
    ("256x256", False, True): [(324, 3712, 3576), (323, 3568, 4040), (349, 3580, 3595)],
    ("256x256", True, False): [(12550, 1984, 2080), (12969, 2312, 1672), (12867, 1946, 2196)],
    ("256x256", True, True): [(8203, 2048, 2080), (7889, 1704, 2360), (7933, 2047, 2099)],
    ("128x256", False, False): [(4466, 2048, 2128), (4247, 1936, 2160), (4131, 2033, 2080)],
    ("128x256", False, True): [(603, 1984, 2104), (596, 2200, 2192), (583, 2153, 2105)],
    ("128x256", True, False): [(8431, 1600, 1680), (8943, 1576, 1800), (8597, 1674, 1551)],
    ("128x256", True, True): [(4524, 1536, 1288), (4120, 1360, 1480), (4134, 1431, 1347)],
    ("128x128 deep", False, True): [(206, 1344, 1312), (203, 1296, 1320), (206, 1860, 1843)],
    ("128x128 deep", True, True): [(1703, 832, 1232), (1868, 1064, 984), (1628, 918, 1114)],
    ("128x128", False, True): [(211, 2112, 2024), (203, 2152, 2000), (201, 2311, 1832)],
    ("128x128", True, True): [(5951, 1664, 1560), (5594, 1808, 1328), (5947, 1605, 1538)],
    ("64x64", False, True): [(202, 64, 72), (204, 72, 72), (210, 69, 65)],
    ("64x64", True, True): [(1360, 64, 72), (1374, 72, 72), (1399, 70, 65)],
    ("64x64 any", False, True): [None, None, (202, 1160, 929)],
    ("64x64 any", True, True): [None, None, (4080, 217, 117)],
}
# the kernel for few rows, on 4, 8 and 16 waves: its unrolled loop taken once to sixteen times a wave
ROWS = [(1, 16336, 11736), (5, 16272, 11336), (12, 1801, 3562), (16, 1800, 8), (9, 1803, 11), (16, 769, 9),
        (1, 15968, 6952), (2, 16120, 7992), (9, 3600, 24), (16, 3640, 2792), (1, 3622, 2447), (2, 3844, 3503),
        (9, 2051, 2865), (1, 16056, 3320), (5, 15384, 3864), (12, 4424, 2696), (1, 4143, 3526)]


def sizes(table):
    """(m, k, n, whether results are whole lines) of every entry."""
    return [(*s, i == 0) for three in table.values() for i, s in enumerate(three) if s is not None]
