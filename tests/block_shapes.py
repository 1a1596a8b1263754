"""Sizes of tests that mean to reach a certain kernel of the feed-forward block or the softmax loss, with the kernels that
have to come out.  tests/test_block_plans_cpu.py holds them against the library's own choice, so that a change of a rule
cannot take a kernel out of the GPU tests unnoticed."""

# (tokens, d, f): serving with a residual, training, backward.  Odd token counts, d and f that end inside tiles.
FFN = {
    (5, 480, 1376): (dict(hidden="rows", out="rows"), dict(hidden="rows", out="rows"), dict(dpre="128x128", together="1")),
    (701, 480, 1376): (dict(hidden="128x128", out="rows"), dict(hidden="128x128", out="rows"), dict(together="1")),
    (127, 1024, 2848): (dict(hidden="rows", out="128x128/10"), dict(hidden="rows", out="128x128/10"), dict(together="1")),
    (12001, 480, 1376): (dict(hidden="256x256", out="128x128"), dict(hidden="128x128", out="128x128"),
                         dict(dpre="128x128", together="0", dx="128x128", dw_in="256x256/10", dw_out="128x128/10")),
    # all on 256 x 256 tiles: h (55 MB) and dpre (110 MB) left in the caches
    (20001, 480, 1376): (dict(hidden="256x256", h="cached", out="256x256"), dict(hidden="256x256", h="cached", out="256x256"),
                         dict(dpre="256x256", store="cached", dx="256x256", dw_in="256x256/10", dw_out="256x256/20")),
    # the second product of a training forward on 256 x 128 tiles
    (40001, 512, 1408): (dict(hidden="256x256", h="cached", out="256x256"), dict(hidden="256x256", h="cached", out="256x128"),
                         dict(dpre="256x256", store="cached", dx="256x256")),
    # h (206 MB) and dpre (413 MB) stored past the caches
    (75001, 480, 1376): (dict(hidden="256x256", h="streamed", out="256x256"), dict(hidden="256x256", h="streamed"),
                         dict(dpre="256x256", store="streamed", dx="256x256", dw_in="256x256/10", dw_out="256x256/20")),
}
# pre and dpre of 2.25e9 elements on 256 x 256 tiles
FFN_LONG = (800_003, 512, 1408)
FFN_LONG_KERNELS = (dict(hidden="256x256", h="streamed"), dict(hidden="256x256", out="256x256"),
                    dict(dpre="256x256", store="streamed", dx="256x256", dw_in="256x256/32"))

# (rows, classes, d, rows with a label): forward, backward
LOSS = {
    # dz of the register tiles past the caches (240 MB); dx and dW on split 256 x 256 tiles
    (10001, 12001, 256, 9900): (dict(logits="registers", run="15"), dict(dz="streamed", dx="256x256/6", dw="256x256/5")),
    # logits on 256 x 256 tiles, dz left in the caches
    (3001, 30011, 288, 3001): (dict(logits="256x256"), dict(logits="256x256", dz="cached", dx="256x256/10", dw="256x256/direct")),
    # two pieces, the second one smaller, dx on 256 x 256 tiles added up over them: several m blocks of rows; one m block
    # and 64 splits, of which 59 have k; dW split over rows, all splits with rows and only the first
    (40001, 60000, 288, 4000): (dict(logits="256x256", pieces="1"), dict(pieces="2", dz="streamed", dx="256x256/8", dw="256x256/direct")),
    (40001, 60000, 288, 200): (dict(logits="256x256"), dict(pieces="2", dz="cached", dx="256x256/64", dw="256x256/direct")),
    (60001, 50011, 320, 2000): (dict(logits="256x256"), dict(pieces="2", dz="cached", dx="256x256/16", dw="256x256/5")),
    (60001, 50011, 320, 60): (dict(logits="256x256"), dict(pieces="2", dx="256x256/64", dw="256x256/5")),
}
# An item's statistics carried over several class tiles: the register tiles, whose items have consecutive tiles of 64
# classes, and the 256 x 256 tiles, whose items have every 66th tile of 256.
CARRIED_REGISTERS = (2501, 20000, 256)
CARRIED_WIDE = (20001, 50011, 288)
CARRIED_RUN = {CARRIED_REGISTERS: 7, CARRIED_WIDE: 3}
