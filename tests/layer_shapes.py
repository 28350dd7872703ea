"""Products and layers for every way that a product can take, with that way: (kernel, pieces of k).  A refit of the estimate that
moves one of them is seen on the host (test_layer_plans.py); the results are checked on the GPU (test_gpu_layer_plans.py)."""
FEW, TILE64_DEEP, TILE64, TILE128, TILE128X64, TILE256, SHALLOW = range(7)

# (M, N, K): kernel, pieces; results four to a thread of the join and one
IN_PIECES = {
    (1, 6088, 265_208): (FEW, 3), (1, 8198, 131_012): (FEW, 2), (8, 8352, 132_341): (FEW, 2),
    (202, 256, 4111): (TILE64_DEEP, 4), (33, 71, 20_000): (TILE64_DEEP, 16),
    (708, 1364, 9174): (TILE128, 4), (1397, 733, 9549): (TILE128, 4),
    (389, 584, 13_132): (TILE128X64, 8), (782, 257, 12_088): (TILE128X64, 8),
    (1090, 1800, 11_645): (TILE256, 4), (963, 1037, 21_878): (TILE256, 8),
}

# (tokens, outputs, inputs): the kernels of dx (tokens x inputs, outputs deep) and dw (outputs x inputs, tokens deep), both in one
# piece and one launch
PAIRS = {
    (669, 656, 33): (TILE64_DEEP, TILE64_DEEP), (33, 681, 40): (TILE64_DEEP, TILE64), (33, 33, 20): (TILE64, TILE64),
    (461, 669, 8237): (TILE128, TILE128), (268, 306, 6780): (TILE128X64, TILE128X64), (1644, 1628, 7895): (TILE256, TILE256),
    (60, 64, 40_000): (SHALLOW, SHALLOW),
}

# (tokens, outputs, inputs): kernel and pieces of dx, and of dw; where both are in pieces they share the workspace
BACKWARD_IN_PIECES = {
    (6277, 6374, 31): ((TILE64_DEEP, 2), (TILE64_DEEP, 2)), (6273, 6436, 32): ((TILE64_DEEP, 2), (TILE64_DEEP, 2)),
    (8222, 4452, 1): ((TILE64_DEEP, 1), (TILE128X64, 7)), (82, 8657, 8211): ((TILE128, 4), (TILE128, 1)),
    (8813, 3513, 1178): ((TILE256, 1), (TILE256, 2)), (5456, 33, 410): ((SHALLOW, 1), (TILE64_DEEP, 4)),
}
