"""Sizes of products that the widest tiles take, and which kernel that is: shared by
the test that runs them on a GPU and the one that asks the rule on the CPU."""

# rows, columns, sum: unsplit with odd rows and with rows in fours; split with rows in fours and odd
SHAPES = [(2047, 8190, 100), (2048, 8191, 585), (2500, 1027, 20000), (131, 8190, 8200), (1501, 2053, 20003)]

# left operands: Source of the rule, and bfloat16 parts
SOURCES = {"mx4": 0, "mx8": 1, "bf16": 2, "f16": 3, "f32": 4}
PARTS = {"mx4": 1, "mx8": 1, "bf16": 1, "f16": 2, "f32": 3}


def kernel(src, op, bbits, m, plan):
    """A product's kernel from its plan (variant, bm, bn, splits): variant, tile, whether the
    left operand is transposed, whether its last lane may lack rows, and whether the sum is split."""
    variant, bm, bn, splits = plan
    turned = op == "T"
    return (src, bbits, variant, bm, bn, turned, turned and m % (bm // 64) != 0, splits > 1)
