"""Sizes of products of 4-bit layers that between them take every form of the kernel that works on tiles (found by planning millions of calls without
a GPU: a plan depends on sizes, types and flags alone).  test_mx_shapes.py holds them to that."""

# (type, quantize, matrices (0: the product that is not grouped), n, m, rows)   # template arguments of mx_tile_kernel; + where the columns' k is split
TILES = [
    ("bfloat16", True, 0, 1029, 588, 913),  # 0, false, __bf16, 2, 1
    ("bfloat16", True, 0, 8539, 136, 398),  # 0, false, __bf16, 2, 1 +
    ("bfloat16", True, 0, 515, 585, 1725),  # 0, false, __bf16, 2, 2
    ("bfloat16", True, 0, 8288, 66, 1324),  # 0, false, __bf16, 2, 2 +
    ("bfloat16", True, 0, 513, 900, 1108),  # 0, false, __bf16, 4, 1
    ("bfloat16", True, 0, 10779, 599, 136),  # 0, false, __bf16, 4, 1 +
    ("bfloat16", True, 0, 323, 645, 2517),  # 0, false, __bf16, 4, 2
    ("bfloat16", True, 0, 16474, 66, 1516),  # 0, false, __bf16, 4, 2 +
    ("bfloat16", True, 0, 302, 134, 17554),  # 0, false, __bf16, 4, 4
    ("bfloat16", True, 0, 312, 4782, 772),  # 0, false, __bf16, 8, 2
    ("bfloat16", True, 0, 306, 1318, 12412),  # 0, false, __bf16, 8, 4
    ("float32", True, 0, 4146, 196, 388),  # 0, false, float, 2, 1
    ("float32", True, 0, 5760, 194, 339),  # 0, false, float, 2, 1 +
    ("float32", True, 0, 648, 716, 1204),  # 0, false, float, 2, 2
    ("float32", True, 0, 8320, 72, 1306),  # 0, false, float, 2, 2 +
    ("float32", True, 0, 664, 526, 1730),  # 0, false, float, 4, 1
    ("float32", True, 0, 14400, 514, 133),  # 0, false, float, 4, 1 +
    ("float32", True, 0, 400, 644, 2221),  # 0, false, float, 4, 2
    ("float32", True, 0, 24960, 258, 725),  # 0, false, float, 4, 2 +
    ("float32", True, 0, 323, 132, 14258),  # 0, false, float, 4, 4
    ("float32", True, 0, 320, 260, 10073),  # 0, false, float, 8, 2
    ("float32", True, 0, 329, 21912, 266),  # 0, false, float, 8, 4
    ("bfloat16", False, 0, 2365, 516, 1300),  # 1, false, __bf16, 2, 1
    ("bfloat16", False, 0, 6501, 395, 853),  # 1, false, __bf16, 2, 1 +
    ("bfloat16", False, 0, 1443, 900, 961),  # 1, false, __bf16, 2, 2
    ("bfloat16", False, 0, 8987, 344, 435),  # 1, false, __bf16, 2, 2 +
    ("bfloat16", False, 0, 791, 1189, 1511),  # 1, false, __bf16, 2, 4
    ("bfloat16", False, 0, 6817, 389, 772),  # 1, false, __bf16, 2, 4 +
    ("bfloat16", False, 0, 655, 1541, 1107),  # 1, false, __bf16, 4, 2
    ("bfloat16", False, 0, 12379, 260, 813),  # 1, false, __bf16, 4, 2 +
    ("bfloat16", False, 0, 445, 1308, 2497),  # 1, false, __bf16, 4, 4
    ("bfloat16", False, 0, 10263, 392, 1145),  # 1, false, __bf16, 4, 4 +
    ("bfloat16", False, 0, 515, 788, 4323),  # 1, false, __bf16, 8, 2
    ("bfloat16", False, 0, 408, 100, 4008),  # 1, true, __bf16, 2, 1
    ("bfloat16", False, 0, 7984, 8, 16),  # 1, true, __bf16, 2, 1 +
    ("bfloat16", False, 0, 392, 354, 2170),  # 1, true, __bf16, 2, 2
    ("bfloat16", False, 0, 7784, 99, 363),  # 1, true, __bf16, 2, 2 +
    ("bfloat16", False, 0, 416, 388, 3574),  # 1, true, __bf16, 2, 4
    ("bfloat16", False, 0, 6272, 132, 1104),  # 1, true, __bf16, 2, 4 +
    ("bfloat16", False, 0, 664, 134, 4411),  # 1, true, __bf16, 4, 1
    ("bfloat16", False, 0, 4224, 17, 1794),  # 1, true, __bf16, 4, 1 +
    ("bfloat16", False, 0, 536, 257, 4775),  # 1, true, __bf16, 4, 2
    ("bfloat16", False, 0, 12544, 276, 727),  # 1, true, __bf16, 4, 2 +
    ("bfloat16", False, 0, 408, 776, 3927),  # 1, true, __bf16, 4, 4
    ("bfloat16", False, 0, 14896, 135, 1057),  # 1, true, __bf16, 4, 4 +
    ("bfloat16", False, 0, 328, 260, 8735),  # 1, true, __bf16, 8, 2
    ("float32", False, 0, 1152, 578, 2233),  # 3, false, float, 2, 2
    ("float32", False, 0, 9066, 598, 311),  # 3, false, float, 2, 2 +
    ("float32", False, 0, 1080, 644, 2262),  # 3, false, float, 2, 4
    ("float32", False, 0, 2392, 707, 1107),  # 3, false, float, 2, 4 +
    ("float32", False, 0, 516, 325, 12026),  # 3, false, float, 4, 2
    ("float32", False, 0, 10707, 324, 821),  # 3, false, float, 4, 2 +
    ("float32", False, 0, 6872, 4417, 33),  # 3, false, float, 4, 4 +
    ("bfloat16", True, 2, 1025, 468, 1199),  # 0, false, __bf16, 2, 1
    ("bfloat16", True, 2, 8645, 132, 371),  # 0, false, __bf16, 2, 1 +
    ("bfloat16", True, 2, 643, 322, 2752),  # 0, false, __bf16, 2, 2
    ("bfloat16", True, 2, 8712, 70, 1333),  # 0, false, __bf16, 2, 2 +
    ("bfloat16", True, 11, 133, 4050, 551),  # 0, false, __bf16, 2, 4
    ("bfloat16", True, 2, 647, 548, 1714),  # 0, false, __bf16, 4, 1
    ("bfloat16", True, 2, 13389, 139, 1252),  # 0, false, __bf16, 4, 1 +
    ("bfloat16", True, 3, 337, 514, 2988),  # 0, false, __bf16, 4, 2
    ("bfloat16", True, 3, 16640, 65, 1419),  # 0, false, __bf16, 4, 2 +
    ("bfloat16", True, 2, 321, 134, 17415),  # 0, false, __bf16, 4, 4
    ("bfloat16", True, 2, 304, 275, 15611),  # 0, false, __bf16, 8, 2
    ("bfloat16", True, 2, 324, 1332, 13039),  # 0, false, __bf16, 8, 4
    ("float32", True, 2, 1200, 261, 1598),  # 0, false, float, 2, 1
    ("float32", True, 2, 5659, 130, 464),  # 0, false, float, 2, 1 +
    ("float32", True, 2, 659, 516, 1638),  # 0, false, float, 2, 2
    ("float32", True, 4, 11198, 67, 646),  # 0, false, float, 2, 2 +
    ("float32", True, 3, 303, 6356, 247),  # 0, false, float, 2, 4
    ("float32", True, 2, 669, 268, 2929),  # 0, false, float, 4, 1
    ("float32", True, 2, 17624, 136, 1187),  # 0, false, float, 4, 1 +
    ("float32", True, 2, 387, 263, 4882),  # 0, false, float, 4, 2
    ("float32", True, 2, 19610, 65, 1647),  # 0, false, float, 4, 2 +
    ("float32", True, 3, 301, 132, 14562),  # 0, false, float, 4, 4
    ("float32", True, 3, 308, 259, 10379),  # 0, false, float, 8, 2
    ("bfloat16", False, 2, 2555, 489, 1373),  # 1, false, __bf16, 2, 1
    ("bfloat16", False, 2, 1421, 593, 1641),  # 1, false, __bf16, 2, 2
    ("bfloat16", False, 2, 5977, 352, 1001),  # 1, false, __bf16, 2, 2 +
    ("bfloat16", False, 2, 827, 728, 2574),  # 1, false, __bf16, 2, 4
    ("bfloat16", False, 2, 7305, 393, 980),  # 1, false, __bf16, 2, 4 +
    ("bfloat16", False, 2, 709, 1060, 1753),  # 1, false, __bf16, 4, 2
    ("bfloat16", False, 2, 12441, 280, 793),  # 1, false, __bf16, 4, 2 +
    ("bfloat16", False, 2, 389, 1040, 3216),  # 1, false, __bf16, 4, 4
    ("bfloat16", False, 2, 10513, 208, 2657),  # 1, false, __bf16, 4, 4 +
    ("bfloat16", False, 2, 573, 541, 5795),  # 1, false, __bf16, 8, 2
    ("bfloat16", False, 2, 440, 97, 4159),  # 1, true, __bf16, 2, 1
    ("bfloat16", False, 2, 7928, 36, 411),  # 1, true, __bf16, 2, 1 +
    ("bfloat16", False, 2, 400, 452, 1733),  # 1, true, __bf16, 2, 2
    ("bfloat16", False, 2, 7856, 68, 424),  # 1, true, __bf16, 2, 2 +
    ("bfloat16", False, 3, 304, 132, 8843),  # 1, true, __bf16, 2, 4
    ("bfloat16", False, 2, 6416, 155, 1045),  # 1, true, __bf16, 2, 4 +
    ("bfloat16", False, 2, 696, 130, 4341),  # 1, true, __bf16, 4, 1
    ("bfloat16", False, 2, 4544, 17, 1931),  # 1, true, __bf16, 4, 1 +
    ("bfloat16", False, 2, 472, 266, 5346),  # 1, true, __bf16, 4, 2
    ("bfloat16", False, 2, 6176, 65, 3242),  # 1, true, __bf16, 4, 2 +
    ("bfloat16", False, 2, 424, 530, 5909),  # 1, true, __bf16, 4, 4
    ("bfloat16", False, 2, 8704, 140, 2383),  # 1, true, __bf16, 4, 4 +
    ("bfloat16", False, 2, 368, 259, 8421),  # 1, true, __bf16, 8, 2
    ("float32", False, 2, 1114, 453, 2813),  # 3, false, float, 2, 2
    ("float32", False, 2, 10942, 327, 890),  # 3, false, float, 2, 2 +
    ("float32", False, 2, 898, 456, 3582),  # 3, false, float, 2, 4
    ("float32", False, 2, 1936, 664, 1595),  # 3, false, float, 2, 4 +
    ("float32", False, 2, 152, 322, 32089),  # 3, false, float, 4, 2
]
