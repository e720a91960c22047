"""Sizes at which the matrix kernels take whole 256 x 256 tiles over more than one 128-byte step of k, and what the library is to plan for them
(tests/test_tile_plans_host.py holds it to that, tests/test_gpu_whole_tiles.py runs them).

A plan is (kind, whole, workgroups, parts): tiles of 128 or 256 rows and columns, how many are taken whole, by how many workgroups, and how many quarters of
cut ones there are beside them."""

# tokens, channels: the plan.  Codes a row: two steps and three, nine, last ones that are short, rows that are not aligned
HEAD = {
    (3000, 3000): (256, 144, 144, 0),
    (4300, 4200): (256, 256, 256, 132),    # a cut last round beside a whole one
    (5000, 6300): (256, 500, 256, 0),      # workgroups of one tile and of two
    (2100, 20_000): (256, 711, 256, 0),    # of two and of three
    (512, 20_000): (256, 158, 158, 0),     # rows are staged through registers (those that are not aligned)
}
HEAD_K = [256, 384, 400, 1152, 1168, 250, 1001]

# tokens, vocabulary: the plan (of the loss, and of the gradient's G, one tile a workgroup)
LOSS = {
    (3000, 3000): (256, 144, 144, 0),
    (4300, 4200): (256, 256, 256, 132),
    (512, 20_000): (256, 158, 158, 0),
}
LOSS_D = [128, 192, 200, 576, 101]

# tokens, vocabulary, width: rows of a piece, workgroups that share a tile of dH; plans of G, of dH and of dW for the first piece
GRAD = {
    (760, 33_000, 744): (33_024, 28, (256, 387, 387, 0), (256, 9, 9, 0), (256, 387, 256, 0)),
    (5000, 50_000, 1000): (25_088, 3, (256, 1960, 1960, 0), (256, 80, 80, 0), (256, 392, 256, 0)),   # two pieces, added
    (40_000, 8200, 440): (2816, 1, (256, 1727, 1727, 0), (256, 256, 256, 232), (256, 0, 0, 88)),     # three pieces
    (3000, 33_000, 1000): (33_024, 5, (256, 1536, 1536, 48), (256, 48, 48, 0), (256, 512, 256, 16)),
    (2000, 50_001, 1024): (50_176, 8, (256, 1536, 1536, 128), (256, 32, 32, 0), (256, 768, 256, 64)),
}
