"""Shapes of the tests of 8-bit products, and what they are to reach: the GPU tests compute
them, a test without a GPU asks which kernels they launch.  Rows, experts, N, K."""

# few rows of each expert: one, two and four tiles of 16 of rows and of columns
FEW = [(1, 1, 1, 1), (1, 1, 300, 77), (3, 1, 65, 128), (16, 1, 4096, 200), (16, 1, 20000, 130), (7, 3, 129, 16),
       (40, 20, 70, 1100), (300, 30, 1000, 257), (9, 1, 33, 5000), (30, 1, 9000, 130), (60, 1, 130, 1030),
       (60, 1, 18000, 1030), (30, 1, 18000, 130), (60, 1, 9000, 130), (5, 1, 10000, 130), (30, 1, 200, 1030)]
# on tiles of 128 and 256, K in whole and broken k-blocks and chunks
SHAPES = [(17, 1, 128, 16), (130, 1, 130, 48), (200, 2, 257, 112), (300, 3, 100, 128), (260, 1, 513, 144),
          (500, 4, 128, 240), (1000, 3, 300, 256), (700, 7, 200, 272), (129, 1, 1000, 1040), (2000, 5, 1024, 400),
          (4100, 3, 1500, 640), (3000, 40, 520, 384), (900, 2, 1500, 2064)]
# on copies of the operands
ODD = [(100, 1, 130, 1), (300, 3, 257, 77), (1000, 5, 129, 1001), (2500, 2, 700, 333), (5000, 4, 700, 333), (4000, 2, 1000, 1001)]
# more tiles than workgroups
LARGE = [(33000, 3, 1030, 144), (20000, 70, 2048, 128), (16000, 1, 4100, 400)]
# long reductions of few tiles, in splits
SPLIT = [(3, 1, 40, 30001), (20, 1, 30, 21600), (39, 1, 64, 6656), (50, 1, 33, 40007), (294, 1, 300, 8128),
         (130, 1, 260, 20016)]
