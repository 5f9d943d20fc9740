"""Sizes that take each way through the training attention's launches, and which one
that is.  Imported only by tests: the CPU suite checks the ways against the library's
rules, the GPU suite runs the sizes."""

# heads, n, d, dtype, c_q, keep, pattern
# bf16 kernels by queries on the block order, in one part, slots cut into halves
ORDERED = [
    (3, 16400, 128, "bf16", 60, 0.3, "uncovered"),
    (4, 16400, 64, "bf16", 60, 0.3, "empty"),
    (2, 16390, 128, "bf16", 300, 0.1, ""),      # most slots hold two clusters
    (16, 4352, 128, "bf16", 1, 1.0, ""),        # dense, whole chunks
    (33, 4100, 64, "bf16", 1, 1.0, ""),         # dense, a ragged last chunk
]
# slots listed by cost, without a block order
BY_COST = [(9, 9000, 64, "bf16", 40, 0.2, "")]
# the same, the lists cut into parts
BY_COST_PARTS = [(40, 700, 128, "bf16", 20, 0.5, ""), (1, 9000, 128, "bf16", 300, 0.1, "empty")]
# chunks listed with the call's preparation, lists cut into parts
LISTED_PARTS = [(1, 4500, 128, "bf16", 1, 1.0, ""), (3, 2185, 128, "bf16", 32, 0.5, "empty")]
# long sequences: heads, n, d, dtype, c_q, keep, dropout
LONG = [
    (1, 118800, 64, "bf16", 40, 0.15, 0.0),     # a block order, keys by signature
    (1, 118800, 128, "f32", 24, 0.1, 0.0),
    (1, 118800, 64, "bf16", 1, 1.0, 0.1),       # dense
    (5, 118800, 128, "bf16", 24, 0.1, 0.1),     # too much K and V for a block order
]
