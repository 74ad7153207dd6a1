"""Shapes of linear layers by the kernels that their passes take, for the tests of these kernels: on the host a test holds the library's plan against
them, so that a rule that moves does not leave a kernel without its test."""

# M, K, N of bf16 layers whose three products all take tiles of 256: steps of 64 in odd and even numbers, ends inside a step, a tile and a half of one
LARGE = [(3080, 2872, 3128), (3064, 2936, 2936), (2824, 2824, 2824)]

# Every other kernel of the products, whole and with a k cut in parts that a launch joins: type, pass (CG_PASS_*), whether bf16 rows are whole 16 bytes, x
# in 8 bits, tile, k cut, and M, K, N: with outputs of few columns or rows (k in the most parts), and near a square.
PRODUCTS = [
    ("bf16", 0, False, False, 64, False, (37, 21, 21), (62, 62, 61)),
    ("bf16", 0, False, False, 64, True, (40, 1031, 23), (527, 2052, 529)),
    ("bf16", 0, False, False, 128, False, (67, 21, 8786), (1739, 1533, 1450), (796, 21, 4770), (2242, 885, 1938)),
    ("bf16", 0, False, False, 128, True, (4231, 1767, 20), (970, 3257, 1098), (8490, 2636, 20), (1578, 4426, 1535)),
    ("bf16", 0, True, False, 64, False, (35, 24, 24), (89, 88, 88)),
    ("bf16", 0, True, False, 64, True, (34, 1096, 24), (467, 1880, 488)),
    ("bf16", 0, True, False, 128, False, (67, 24, 8904), (1406, 1464, 1832), (8641, 24, 440), (1910, 792, 2184)),
    ("bf16", 0, True, False, 128, True, (67, 2120, 3032), (1367, 3432, 712), (4728, 5768, 24), (1448, 4136, 1528)),
    ("bf16", 1, False, False, 64, False, (37, 21, 21), (62, 62, 61)),
    ("bf16", 1, False, False, 64, True, (34, 20, 1094), (494, 477, 1906)),
    ("bf16", 1, False, False, 128, False, (65, 8362, 23), (1456, 1517, 1274), (8416, 396, 20), (1665, 2310, 940)),
    ("bf16", 1, False, False, 128, True, (4228, 20, 2556), (1265, 831, 3281), (5489, 22, 2028), (1648, 1518, 4401)),
    ("bf16", 1, True, False, 64, False, (35, 24, 24), (89, 88, 88)),
    ("bf16", 1, True, False, 64, True, (38, 24, 1048), (441, 440, 1768)),
    ("bf16", 1, True, False, 128, False, (8443, 72, 24), (1609, 1288, 1192), (425, 8264, 24), (1630, 2488, 984)),
    ("bf16", 1, True, False, 128, True, (5558, 24, 2088), (1000, 1032, 3864), (6594, 24, 3352), (1451, 1416, 3992)),
    ("bf16", 2, False, False, 64, False, (37, 21, 21), (62, 62, 61)),
    ("bf16", 2, False, False, 64, True, (1064, 22, 20), (2186, 565, 553)),
    ("bf16", 2, False, False, 128, False, (33, 76, 8290), (1739, 1533, 1450), (33, 643, 5726), (963, 1749, 2371)),
    ("bf16", 2, False, False, 128, True, (1731, 4436, 22), (3362, 902, 1107), (4683, 20, 4130), (4033, 6638, 149)),
    ("bf16", 2, False, True, 64, False, (37, 21, 21), (62, 62, 61)),
    ("bf16", 2, False, True, 64, True, (1064, 22, 20), (2186, 565, 553)),
    ("bf16", 2, False, True, 128, False, (33, 76, 8290), (1739, 1533, 1450), (33, 643, 5726), (963, 1749, 2371)),
    ("bf16", 2, False, True, 128, True, (1731, 4436, 22), (3362, 902, 1107), (4683, 20, 4130), (4033, 6638, 149)),
    ("bf16", 2, True, False, 64, False, (35, 24, 24), (89, 88, 88)),
    ("bf16", 2, True, False, 64, True, (1038, 24, 24), (1839, 440, 472)),
    ("bf16", 2, True, False, 128, False, (37, 72, 8872), (1255, 1576, 1400), (33, 664, 5432), (886, 2072, 2072)),
    ("bf16", 2, True, False, 128, True, (2657, 24, 4168), (3502, 1176, 968), (2841, 6712, 24), (4729, 1464, 1688)),
    ("bf16", 2, True, True, 64, False, (35, 24, 24), (89, 88, 88)),
    ("bf16", 2, True, True, 64, True, (1038, 24, 24), (1839, 440, 472)),
    ("bf16", 2, True, True, 128, False, (37, 72, 8872), (1255, 1576, 1400), (33, 664, 5432), (886, 2072, 2072)),
    ("bf16", 2, True, True, 128, True, (2657, 24, 4168), (3502, 1176, 968), (2841, 6712, 24), (4729, 1464, 1688)),
    ("fp32", 0, False, False, 64, False, (40, 20, 20), (82, 84, 83)),
    ("fp32", 0, False, False, 64, True, (33, 364, 26), (455, 475, 429)),
    ("fp32", 0, False, False, 128, False, (8413, 20, 67), (1935, 1247, 1539)),
    ("fp32", 0, False, False, 128, True, (2085, 1351, 69), (1470, 1463, 1515)),
    ("fp32", 1, False, False, 64, False, (40, 20, 20), (82, 84, 83)),
    ("fp32", 1, False, False, 64, True, (37, 20, 380), (523, 511, 524)),
    ("fp32", 1, False, False, 128, False, (8710, 67, 21), (1735, 1901, 1207)),
    ("fp32", 1, False, False, 128, True, (65, 2874, 654), (1470, 1463, 1515)),
    ("fp32", 2, False, False, 64, False, (40, 20, 20), (82, 84, 83)),
    ("fp32", 2, False, False, 64, True, (412, 20, 21), (523, 511, 524)),
    ("fp32", 2, False, False, 128, False, (37, 8387, 75), (1105, 1842, 1754)),
    ("fp32", 2, False, False, 128, True, (667, 67, 2749), (1470, 1463, 1515)),
    ("fp32", 2, False, True, 64, False, (40, 20, 20), (82, 84, 83)),
    ("fp32", 2, False, True, 64, True, (412, 20, 21), (523, 511, 524)),
    ("fp32", 2, False, True, 128, False, (37, 8387, 75), (1105, 1842, 1754)),
    ("fp32", 2, False, True, 128, True, (667, 67, 2749), (1470, 1463, 1515)),
]
CASES = [(*p[:6], *shape) for p in PRODUCTS for shape in p[6:]]
