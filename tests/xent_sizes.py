"""Sizes at which the loss is compared with its definition: tokens, classes, channels.
test_xent_kernels_on_cpu.py makes the same calls of the launchers compiled for the host,
and fails where they leave a kernel out."""

F32, BF16, NONE = 0, 1, -1
# types of dx and dw; either may be left out
TYPES = [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)]
ALONE = [(F32, NONE), (NONE, F32), (BF16, NONE), (NONE, BF16)]

SMALL = [(1, 1, 1), (1, 2, 3), (3, 1, 64), (2, 100, 16), (1, 257, 130), (5, 33, 17), (16, 100, 384),
         (17, 130, 129), (31, 64, 128), (33, 65, 200), (63, 1000, 63), (64, 1001, 384),
         (65, 2, 400), (65, 100, 384), (66, 127, 127), (100, 129, 128), (128, 100, 384),
         (127, 256, 255), (129, 255, 257), (200, 513, 100)]
MIDDLE = [(1, 5003, 515), (7, 20011, 130), (31, 3001, 1030), (65, 4099, 700), (255, 2049, 385),
          (257, 4000, 64), (400, 1500, 1111), (997, 1235, 385), (1023, 515, 130), (1030, 3001, 40),
          (2051, 1003, 259), (3001, 70, 300), (515, 9001, 131), (1, 40001, 33)]
# the last ones: several pieces of the classes
LARGE = [(1000, 12345, 385), (2100, 8200, 515), (4099, 2051, 1030), (300, 32003, 257),
         (8200, 1003, 131), (997, 70001, 70), (4100, 20001, 100), (9001, 9001, 65),
         (33, 300007, 40)]
