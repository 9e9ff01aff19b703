"""Products grouped by expert that reach every kernel they may run on, each with the plan it is there for.

A case is (kind, rows of the experts, rows of the bound behind them, K, N, plan).  kind: "fwd" rows times weights, "dx" rows times
transposed weights, "mx" the same in 4 bits, "dw" the gradient of the weights.  plan: rows of a tile, is the reduction cut into
ranges, are those of the last round's tiles cut on the device."""

CASES = [
    # few rows, streamed: some experts end inside a tile, some have several
    ("fwd", [1, 0, 1, 0], 0, 1032, 8200, (16, False, False)),
    ("fwd", [17, 0, 3, 5, 0, 1, 0, 2], 0, 520, 2568, (16, False, False)),
    ("fwd", [3, 0, 9], 0, 8264, 72, (16, True, False)),
    ("fwd", [2, 0, 0, 17, 0, 1], 30, 4360, 264, (16, True, False)),
    ("fwd", [40, 3, 0, 33], 0, 200, 264, (32, False, False)),
    ("fwd", [35, 0, 4], 0, 2056, 136, (32, True, False)),
    ("dx", [1, 0, 2], 0, 1264, 1088, (16, False, False)),
    ("dx", [17, 0, 3, 5, 0, 1, 0, 2], 0, 1032, 1288, (16, False, False)),
    ("dx", [2, 0, 17, 1], 0, 16392, 40, (16, True, False)),
    ("dx", [40, 3, 0, 33], 0, 200, 264, (32, False, False)),
    ("dx", [35, 0, 4, 33], 0, 2328, 168, (32, True, False)),
    ("mx", [9, 0, 20], 0, 2912, 40, (16, False, False)),
    ("mx", [1, 0, 17, 2], 0, 46304, 24, (16, True, False)),
    ("mx", [40, 3, 0, 33], 0, 544, 264, (32, False, False)),
    ("mx", [9, 0, 34], 0, 9248, 40, (32, True, False)),
    # tiles of 128 rows; reductions that end inside a step, ranges of unequal length
    ("fwd", [700, 0, 129, 1], 0, 136, 1288, (128, False, False)),
    ("fwd", [838], 0, 3104, 136, (128, True, False)),
    ("fwd", [1500, 0, 77, 900, 0, 1], 200, 3336, 136, (128, True, False)),
    ("dx", [700, 0, 129, 1], 0, 136, 1288, (128, False, False)),
    ("dx", [2500, 0, 1, 1800, 800, 89], 0, 12368, 304, (128, True, False)),
    ("mx", [700, 0, 129, 1], 0, 288, 1288, (128, False, False)),
    ("mx", [2500, 0, 1, 1800, 800, 89], 0, 12384, 304, (128, True, False)),
    ("mx", [900, 0, 500, 844], 0, 15264, 296, (128, True, False)),
    # tiles of 256 rows: experts that end inside a quarter, odd and even numbers of steps, one step
    ("fwd", [1500, 0, 257, 1100], 0, 552, 3592, (256, False, False)),
    ("fwd", [1300, 0, 1700], 0, 8200, 1000, (256, False, True)),
    ("dx", [1500, 0, 257, 1100], 0, 552, 3592, (256, False, False)),
    ("dx", [2500, 900, 0, 1100], 0, 5128, 4104, (256, False, True)),
    ("mx", [2000, 0, 1800, 1200], 0, 1056, 4104, (256, False, False)),
    ("mx", [2000, 0, 1, 1830, 1100], 400, 1536, 4104, (256, False, False)),
    ("mx", [3001, 0, 900], 0, 160, 4104, (256, False, False)),
    # gradients of weights: experts without rows between others, reductions of unequal length
    ("dw", [33, 0, 250, 64], 0, 200, 264, (128, False, False)),
    ("dw", [3000, 0, 1, 999], 0, 264, 24, (128, True, False)),
    ("dw", [700, 0, 1, 260, 640], 0, 2056, 2064, (256, False, False)),
    ("dw", [63, 129, 0, 65, 400], 100, 2312, 2080, (256, False, False)),
    ("dw", [700, 0, 1, 260, 640], 0, 2056, 2056, (256, False, False)),
]

# every plan that the rules can come to
PLANS = {("fwd", 16, False, False), ("fwd", 16, True, False), ("fwd", 32, False, False), ("fwd", 32, True, False), ("fwd", 128, False, False),
         ("fwd", 128, True, False), ("fwd", 256, False, False), ("fwd", 256, False, True)}
PLANS |= {("dx", *p[1:]) for p in PLANS} | {("mx", *p[1:]) for p in PLANS if not p[3]} | {("dw", *p[1:]) for p in PLANS if p[1] > 32 and not p[3]}
