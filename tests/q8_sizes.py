"""Sizes at which the 8-bit path's operators are compared with their definitions, so that
each of its kernels runs: test_q8_kernels_on_cpu.py asks the launchers which kernels these
calls take, and fails where one is left out (after a change of a rule, say).  The GPU tests
make the same calls.  In a call: storage types 0 (fp32) and 1 (bf16), -1 for none.
"""
from itertools import product

F32, BF16, NONE = 0, 1, -1
TYPES = list(product((F32, BF16), (F32, BF16)))

# T, width: on both sides of 4096 tokens, where a wavefront takes over from a block (a
# last block of rows that is not full among them), and each width's way to hold a row
ROWS = [(4095, 513), (4099, 300), (4099, 513), (4099, 700), (4095, 1024), (4099, 1024),
        (4099, 1025), (4095, 1300), (4099, 1300), (4099, 2047), (4095, 2048), (4099, 2048),
        (37, 1030), (13, 4001), (9, 8001), (6, 16001), (5, 32003), (3, 33001)]

# T, D of the norm's backward pass: two launches, with two or more rows a group and a last
# turn that not all groups have, for each way to hold a row; then one launch
NORM_BWD = [(9001, 384), (4099, 500), (2051, 1030), (3077, 2047), (3077, 4095), (2051, 2050),
            (2100, 8190), (1500, 16000), (1300, 16390), (1023, 130), (300, 700), (60, 4090)]

# M, N, K
PRODUCTS = [(9, 1001, 1300), (20, 333, 1111), (50, 1030, 777),  # few tokens
            (100, 300, 4097), (70, 1000, 4000), (200, 512, 8191), (65, 33, 9000),  # slices
            (150, 1401, 1111), (1576, 1153, 385), (4206, 65, 2011), (2500, 1003, 333),  # 64 x 64
            (777, 3700, 1003),  # 128 x 64 or 128 x 128
            (4403, 222, 643), (3725, 515, 783), (1820, 4279, 1026),
            (1373, 2977, 698),  # 256 x 128
            (2100, 4101, 4109), (2076, 4645, 659)]  # 256 x 256

# T, N, K with the types of dy and of the result
_GRADS = {
    "grad_input": [
        # few tokens, in one piece and in slices
        ((5, 222, 700), TYPES), ((16, 700, 333), TYPES), ((20, 222, 300), TYPES),
        ((32, 1100, 515), TYPES),
        # the 8-bit operand as it lies
        ((66, 3434, 1001), [(BF16, BF16)]), ((35, 692, 130), [(BF16, BF16)]),
        ((66, 3434, 4379), [(BF16, BF16)]), ((128, 704, 4379), [(BF16, BF16)]),
        ((66, 234, 25349), [(BF16, BF16)]), ((68, 201, 54894), [(BF16, BF16)]),
        # laid out: 64 x 64, 128 x 128, 256 x 128, 256 x 256
        ((45, 637, 130), TYPES), ((115, 2444, 130), TYPES), ((2281, 4151, 70), TYPES),
        ((4619, 1124, 100), TYPES), ((33, 1262, 4214), TYPES),
        ((4829, 957, 396), TYPES), ((723, 684, 2807), TYPES), ((2316, 686, 851), TYPES),
        ((2657, 1295, 3029), TYPES), ((1677, 774, 3606), TYPES), ((3338, 611, 1988), TYPES),
        ((2243, 619, 1830), TYPES), ((1917, 625, 4422), TYPES), ((4001, 1031, 4099), TYPES)],
    "grad_weight": [
        # few tokens: narrow and wide tiles
        ((5, 222, 700), TYPES), ((64, 333, 515), TYPES), ((41, 751, 4268), TYPES),
        ((33, 4593, 813), TYPES),
        # both operands as they lie
        ((99, 130, 70), [(BF16, BF16)]), ((102, 1405, 2975), [(BF16, BF16)]),
        ((67, 2491, 1289), [(BF16, BF16)]), ((500, 2047, 2047), [(BF16, BF16)]),
        ((165, 1667, 4461), [(BF16, BF16)]), ((511, 8190, 4095), [(BF16, BF16)]),
        ((1024, 1999, 4301), [(BF16, BF16)]),
        # laid out
        ((801, 130, 70), TYPES), ((4234, 73, 65), TYPES), ((4761, 70, 3044), TYPES),
        ((1061, 130, 70), TYPES), ((4037, 1430, 70), TYPES), ((4174, 70, 2427), TYPES),
        ((882, 667, 3070), TYPES), ((1029, 667, 3070), TYPES), ((649, 2964, 961), TYPES),
        ((601, 684, 3019), TYPES),
        ((3669, 1540, 4815), TYPES), ((729, 3235, 2161), TYPES), ((631, 2982, 3420), TYPES),
        ((610, 4148, 995), TYPES), ((1029, 3099, 3251), TYPES), ((1031, 4001, 4099), TYPES)],
}
GRADS = [(op, *size, *t) for op in _GRADS for size, types in _GRADS[op] for t in types]


def calls():
    """All of them, as tests/native/on_cpu/q8_calls takes them."""
    for T, D in ROWS:
        for x, y in TYPES:
            yield "rows", T, D, x, y
            yield "norm", T, D, x, y, 1, y
            for kind in (0, 1):
                yield "act", kind, T, D, x, y, 1
        for x in (F32, BF16):
            yield "values", T, D, x
            for kind in (0, 1):
                yield "act_bwd", kind, T, D, x
    for T, D in NORM_BWD:
        for a, w in TYPES:
            yield "norm_bwd", T, D, a, w, 1, w
    for s in PRODUCTS:
        for y in (F32, BF16):
            yield "product", *s, y
    yield from GRADS
    # a gradient summed over nothing
    yield "grad_weight", 0, 70, 90, F32, F32
