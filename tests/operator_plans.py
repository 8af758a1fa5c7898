"""Sizes at which every kernel of the products runs: each tile in each direction, its sums whole and split, with every way of the operands into LDS; for the
loss also in one piece and in several (rows stored to where they came from, sums between pieces).  test_operator_plans_host asserts that
they do; test_gpu_operator_plans runs them."""
import paper_1906_12043_amd as P

# groups, rows, inner, outer
PRODUCTS = [
    (1, 16, 64, 64), (2, 16, 519, 519), (1, 9000, 136, 136), (3, 500, 4103, 135), (1, 4000, 64, 2055), (4, 200, 64, 4104), (1, 700, 8200, 136),
    (1, 9000, 520, 520), (1, 700, 136, 16392), (1, 16, 4104, 64), (1, 1500, 8199, 136), (3, 1000, 136, 16392), (1, 3000, 519, 2055), (1, 9000, 4104, 136),
    (8, 700, 263, 16392), (8, 700, 16392, 264), (1, 9000, 136, 8200), (3, 1500, 519, 16392), (3, 1500, 16392, 520)]
# the same with x in codes (weight gradient)
CODES = [(1, 16, 63, 64), (8, 16, 63, 1031), (1, 1000, 63, 64), (8, 16, 519, 519), (3, 9000, 135, 135), (1, 9000, 264, 520), (8, 16, 64, 2056),
         (3, 500, 136, 16392), (1, 6000, 1031, 263), (1, 9000, 136, 8200)]
# groups, rows, dim, vocab, piece
LOSSES = [
    (1, 16, 64, 700, 512), (8, 1000, 135, 700, 512), (3, 500, 135, 4104, 4096), (1, 4000, 64, 300, 0), (2, 200, 136, 8200, 0), (2, 64, 64, 12000, 4096),
    (2, 9000, 135, 300, 0), (1, 200, 263, 2056, 0), (1, 1000, 264, 2056, 2048), (1, 9000, 136, 1500, 1024), (1, 500, 4104, 300, 0), (1, 700, 136, 8200, 0),
    (1, 9000, 263, 700, 512), (2, 3000, 136, 4104, 4096), (1, 2000, 1031, 300, 0), (3, 500, 1031, 4104, 0), (8, 700, 4104, 300, 0), (8, 700, 263, 8200, 8192),
    (8, 700, 4104, 700, 512), (2, 1000, 136, 16400, 0), (1, 9000, 136, 4104, 4096), (1, 1000, 4104, 700, 0), (1, 1000, 4104, 700, 512),
    (8, 700, 264, 16400, 0), (2, 3000, 136, 8200, 8192), (1, 3000, 4104, 300, 0), (1, 6000, 264, 8200, 8192), (1, 3000, 4104, 700, 512), (1, 2000, 264, 24000, 0)]

KINDS = {"bf16": P.BF16, "fp16": P.F16, "fp32": P.F32}
DIRECTIONS = {"forward": P.GROUPED_FORWARD, "input_grad": P.GROUPED_INPUT_GRAD, "weight_grad": P.GROUPED_WEIGHT_GRAD}
LARGE, MEDIUM, SMALL, DEEP, TALL, SQUARE = range(6)
COLUMNS = (256, 128, 64, 128, 128, 64)           # of the tiles
DIRECT, REGISTERS, FROM_CODES = range(3)
A = 1 << 40                                      # addresses that no plan looks behind


def bounds_of(groups, rows):
    """Groups of growing length, the first row and the last one in none, the second of three or more groups empty."""
    cuts = [1 + (rows - 2) * i * i // (groups * groups) for i in range(groups + 1)]
    if groups > 2:
        cuts[2] = cuts[1]
    return cuts


def product_call(dtype, groups, rows, inner, outer, codes=False):
    f = dict(x=None, x_codes=2 * A, ld_codes=inner, x_scales=9 * A, ld_scales=-(-inner // 32)) if codes else dict(x=2 * A, ldx=inner)
    return P.Grouped(dtype=KINDS[dtype], groups=groups, rows=rows, inner=inner, outer=outer, offsets=A, w=3 * A, ldw=outer, w_stride=inner * outer, y=4 * A,
                     ldy=outer, dy=5 * A, lddy=outer, dx=6 * A, lddx=inner, dw=7 * A, lddw=outer, dw_stride=inner * outer, dw_dtype=P.F32, workspace=8 * A,
                     workspace_bytes=1 << 39, **f)


def loss_call(dtype, groups, rows, dim, vocab, piece):
    return P.CrossEntropy(dtype=KINDS[dtype], groups=groups, rows=rows, dim=dim, vocab=vocab, offsets=A, h=2 * A, ldh=dim, e=3 * A, lde=dim,
                          e_stride=vocab * dim, targets=4 * A, loss=5 * A, dh=6 * A, lddh=dim, de=7 * A, ldde=dim, de_stride=vocab * dim, piece=piece,
                          workspace=8 * A, workspace_bytes=1 << 39)


def of_products(dtype, cases=PRODUCTS):
    """{(direction, tile, sums split, operands)} of results that hold a whole tile's columns."""
    out = set()
    for case in cases:
        for kind, direction in DIRECTIONS.items():
            tile, splits, operands = P.debug_grouped_plan(product_call(dtype, *case), direction)
            if (case[2] if kind == "input_grad" else case[3]) >= COLUMNS[tile]:
                out.add((kind, tile, splits > 1, operands))
    return out


def of_codes(dtype, cases=CODES):
    """{(tile, sums split, dy goes to LDS directly)}"""
    out = set()
    for case in cases:
        tile, splits, operands = P.debug_grouped_plan(product_call(dtype, *case, codes=True), P.GROUPED_WEIGHT_GRAD)
        assert operands == FROM_CODES
        if case[3] >= COLUMNS[tile]:
            out.add((tile, splits > 1, dtype != "fp32" and case[3] % 8 == 0))
    return out


def of_losses(dtype, cases=LOSSES):
    """{("logits" or "slopes", tile, operands)}, {("dh", tile, sums split, several pieces, operands)}, {("de", tile, sums split)}"""
    out = set()
    for case in cases:
        (logits, slopes, dh, de), pieces = P.debug_cross_entropy_plan(loss_call(dtype, *case))
        out.add(("logits", logits[0], logits[2]))
        if slopes[1]:
            out.add(("slopes", slopes[0], slopes[2]))
        if case[2] >= COLUMNS[dh[0]]:
            out.add(("dh", dh[0], dh[1] > 1, pieces > 1, dh[2]))
        if case[2] >= COLUMNS[de[0]]:
            out.add(("de", de[0], de[1] > 1))
    return out
