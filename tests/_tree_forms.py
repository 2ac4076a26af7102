"""Sizes of murmur_decode_attn_tree that reach every instance of its kernels: the workgroup's shape and the splits of the
list are the plan's (tests/test_tree_plan.py), the outputs' type the call's."""

FEW, WIDE, PAIR = 0, 1, 2  # eight wavefronts of one or two row tiles each, four of two
# name: (layers, sequences, query heads, KV heads, nodes, longest list), (shape, splits, row sets)
FORMS = {
    "few, whole lists": ((2, 40, 8, 2, 6, 900), (FEW, 1, 1)),
    "few, several splits": ((1, 12, 28, 4, 16, 900), (FEW, 5, 1)),
    "few, many splits": ((1, 1, 28, 4, 5, 9000), (FEW, 64, 1)),
    "wide, whole lists": ((1, 40, 28, 4, 16, 900), (WIDE, 1, 1)),
    "wide, several splits": ((1, 12, 28, 4, 16, 2000), (WIDE, 5, 1)),
    "wide, five row sets": ((1, 12, 16, 1, 40, 2000), (WIDE, 4, 5)),
    "wide, many splits": ((1, 2, 28, 4, 40, 4000), (WIDE, 10, 3)),
    "pair, whole lists": ((1, 24, 28, 4, 40, 300), (PAIR, 1, 3)),
    "pair, several splits": ((2, 6, 28, 4, 40, 900), (PAIR, 3, 3)),
    "pair, one row set": ((1, 24, 28, 4, 16, 2000), (PAIR, 5, 1)),
    "pair, many splits": ((1, 3, 28, 4, 40, 4000), (PAIR, 14, 3)),
}
