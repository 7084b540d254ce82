"""Sizes of the gated feed-forward block at which each kernel instance of its tile products
is the one that the rule picks, with what it picks.

A case: float32 operands or bfloat16, tokens, dim, hidden, then the tiles and splits of the
forward products, of the inner ones of the backward pass, and of dx and of the weights'
gradients: (together in one launch, dx, weights).  L: 256-square, M: 192 x 256, S: 128-square.
"""

CASES = [
    (False, 138, 16, 16, "S1", "S1", (False, "S1", "S1")),
    (False, 34, 736, 16, "S3", "S3", (True, "S1", "S1")),
    (False, 457, 16, 68, "S1", "S1", (True, "S1", "S2")),
    (False, 402, 16, 8481, "M1", "M1", (True, "S16", "S1")),
    (False, 8116, 16, 653, "L1", "L1", (True, "S3", "S16")),
    (False, 4394, 920, 16, "S3", "S3", (True, "L1", "M16")),
    (False, 1994, 3664, 1098, "S1", "S1", (True, "L1", "M1")),
    (False, 921, 673, 7211, "L1", "L1", (True, "L8", "M1")),
    (False, 6676, 155, 6315, "L1", "L1", (True, "L4", "M3")),
    (False, 2332, 2080, 1175, "S1", "S1", (True, "L1", "L1")),
    (False, 2811, 1451, 69, "S5", "S5", (True, "L1", "L11")),
    (False, 130, 1480, 4740, "S3", "S3", (True, "L15", "L1")),
    (False, 2084, 136, 4917, "M1", "M1", (True, "L14", "L3")),
    (False, 5735, 2056, 17, "S7", "S7", (False, "L1", "S15")),
    (False, 5541, 1448, 17, "S5", "S5", (False, "M1", "S15")),
    (False, 8079, 16, 7882, "L1", "L1", (False, "S8", "S4")),
    (False, 1050, 1296, 5266, "M1", "M1", (False, "S5", "L1")),
    (False, 7210, 2776, 408, "S1", "S1", (False, "M1", "L5")),
    (False, 1415, 1744, 3262, "M1", "M1", (False, "S3", "M1")),
    (False, 8247, 1576, 527, "M1", "M1", (False, "L1", "M6")),
    (False, 19833, 136, 3350, "L1", "L1", (False, "L3", "M7")),
    (False, 16093, 136, 3867, "L1", "L1", (False, "M3", "M6")),
    (True, 2328, 2112, 16, "S16", "S16", (False, "S1", "S15")),
    (True, 67, 16, 16, "S1", "S1", (True, "S3", "S3")),
    (True, 65, 16, 910, "S1", "S1", (True, "S15", "S1")),
    (True, 772, 16, 4739, "M1", "M1", (True, "S16", "S2")),
    (True, 6201, 16, 2056, "L1", "L1", (False, "S10", "S15")),
    (True, 8382, 956, 67, "M5", "M5", (True, "S1", "S16")),
    (True, 109, 2152, 16, "S16", "S16", (True, "S1", "S1")),
    (True, 1822, 1448, 16, "S16", "S16", (True, "L1", "L15")),
    (True, 2058, 1315, 18, "S16", "S16", (True, "L1", "M16")),
    (True, 1565, 3760, 1369, "L3", "L3", (True, "L1", "M1")),
    (True, 8585, 1792, 66, "L7", "L7", (False, "L1", "S16")),
    (True, 4119, 1960, 16, "S15", "S15", (False, "M1", "S16")),
    (True, 131, 1784, 1290, "S12", "S12", (True, "L14", "L1")),
    (True, 2146, 2190, 1076, "L3", "L3", (True, "L1", "L1")),
    (True, 3198, 144, 711, "S1", "S1", (True, "L9", "M16")),
    (True, 2584, 690, 205, "S6", "S6", (True, "L3", "L16")),
    (True, 130, 2088, 2199, "S7", "S7", (True, "L12", "M1")),
    (True, 275, 2000, 3526, "S3", "S3", (False, "M16", "L1")),
    (True, 7722, 136, 1885, "L1", "L1", (False, "L8", "L16")),
    (True, 3409, 2120, 138, "S6", "S6", (False, "S1", "M13")),
    (True, 271, 1416, 2684, "S4", "S4", (False, "S14", "S1")),
    (True, 263, 1691, 3077, "M5", "M5", (False, "S12", "M1")),
]
