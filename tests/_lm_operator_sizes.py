"""Sizes at which the operators at the ends of a language model take each of their
kernels, with what they take there: test_lm_operator_plans.py holds the second on
the CPU, the GPU tests run the calls. (bf16: 1, fp32: 0, the types' numbers.)"""

# (type, rows, width, forward's threads a row and vectors a thread) where the layer norm's forward pass takes two rows a thread;
# the last workgroup has one row less
LAYER_TWO_ROWS = [
    (1, 66001, 40, 16, 1), (1, 16403, 260, 64, 1), (1, 16403, 700, 64, 2), (1, 4099, 2048, 256, 1), (1, 4099, 3900, 256, 2),
    (1, 4099, 6000, 1024, 1), (0, 66001, 20, 16, 1), (0, 17001, 300, 64, 2), (0, 4099, 1000, 256, 1), (0, 4099, 2048, 256, 2),
    (0, 4099, 3000, 1024, 1),
]
# (type, rows, width) of rows so wide that a workgroup is one row's, for several rows in turn: shares of dweight and dbias in
# registers, and (above 8192 values) in LDS
LAYER_SHARES = [(1, 1100, 4100), (1, 600, 8190), (1, 600, 8200), (1, 520, 16384), (0, 600, 3000), (0, 600, 6000), (0, 600, 8200),
                (0, 520, 16384)]

# (tokens, vocab, width, the sort's kernels): one workgroup up to 6144 tokens, then by the bits of a digit (9 or 11) and the
# number of digits
EMBED_SORTS = [
    (6144, 600, 36, "one"), (6145, 300, 36, (9, 1)), (6145, 600, 36, (11, 1)), (9000, 511, 12, (9, 1)), (9000, 512, 12, (11, 1)),
    (20000, 1500, 9, (11, 1)), (9000, 2047, 5, (11, 1)), (9000, 2048, 5, (9, 2)), (9000, 262143, 3, (9, 2)), (9000, 262144, 3, (11, 2)),
    (9000, 300000, 3, (11, 2)), (9000, 2000000, 1, (11, 2)), (70001, 300000, 2, (11, 2)), (6145, 4194303, 1, (11, 2)),
    (6145, 4194304, 1, (9, 3)), (600001, 700, 2, (11, 1)),
]

# The losses: (type, rows, width, vocab, columns more that a row of the weights has, elements that it begins late, tiles of
# STATS, GRAD, DX and DW, 1 where the weights
# pass through registers (0: not), pieces of the vocabulary, whether dW is a sum of parts).
# Every product has several blocks of k, and edges that no tile's size divides.
LARGE, MEDIUM, SMALL, TERMS_LARGE, TERMS = (256, 256), (128, 128), (128, 64), (256, 128), (128, 64)
HEADS = [
    (1, 2048, 1024, 32768, 0, 0, (LARGE, LARGE, LARGE, LARGE), [0], 1, False),
    (1, 1999, 1016, 32601, 8, 8, (LARGE, LARGE, LARGE, LARGE), [0], 1, False),
    (1, 4877, 800, 5107, 0, 0, (LARGE, LARGE, LARGE, LARGE), [0], 1, True),
    (1, 8190, 1032, 33001, 0, 0, (LARGE, LARGE, LARGE, MEDIUM), [0], 2, False),
    (1, 6599, 721, 613, 0, 0, (MEDIUM, MEDIUM, MEDIUM, SMALL), [1], 1, True),
    (1, 6599, 728, 613, 5, 1, (MEDIUM, MEDIUM, MEDIUM, SMALL), [1], 1, True),
    (1, 777, 500, 10007, 0, 0, (MEDIUM, MEDIUM, SMALL, MEDIUM), [1], 1, False),
    (1, 67, 2847, 4141, 1, 1, (SMALL, SMALL, SMALL, LARGE), [1], 1, False),
    (1, 68, 2088, 21937, 0, 0, (MEDIUM, MEDIUM, MEDIUM, MEDIUM), [0], 1, False),
    (1, 6740, 136, 2814, 0, 0, (MEDIUM, MEDIUM, SMALL, MEDIUM), [0], 1, True),
    (0, 5061, 624, 1154, 3, 1, (TERMS_LARGE, TERMS_LARGE, TERMS_LARGE, TERMS_LARGE), [0], 1, True),
    (0, 1793, 136, 46041, 0, 0, (TERMS, TERMS_LARGE, TERMS_LARGE, TERMS_LARGE), [0, 1], 2, True),
    (0, 2048, 1024, 32768, 0, 0, (TERMS_LARGE, TERMS_LARGE, TERMS_LARGE, TERMS_LARGE), [0], 1, False),
    (0, 777, 500, 10007, 0, 0, (TERMS, TERMS, TERMS, TERMS), [1], 1, False),
    (0, 71, 1050, 333, 0, 0, (TERMS, TERMS, TERMS, TERMS), [0], 1, False),
]
