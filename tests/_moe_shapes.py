"""Shapes of the tests of large grouped products, and what they are to reach: the GPU
tests compute them, a test without a GPU asks which kernels they launch.  Rows, experts,
N, K; the last tenth of the rows belongs to no expert."""

# tiles of 256 x 256: one for each workgroup at most, or several; last ones partly filled
TILES_256 = [(15872, 2, 1000, 128), (16000, 1, 1024, 320), (31000, 3, 1000, 192), (56000, 70, 512, 128)]
# several tiles of 128 x 128 to a workgroup
TILES_128 = [(20000, 7, 2048, 192), (33000, 70, 1000, 128)]
# the matrices' gradients: more tiles of 256 than workgroups; more of 128
GRADIENTS_256 = [(3000, 64, 1024, 512), (6000, 70, 520, 768), (9000, 20, 1024, 1032)]
GRADIENTS_128 = [(3000, 64, 264, 520), (4000, 200, 120, 384)]
# 4 bits, columns in passes: rows, experts, N, K, group
PASSES = [(5, 1, 140000, 256, 64), (100, 64, 8200, 256, 32), (1000, 40, 12000, 128, 64), (1700, 40, 12001, 256, 128),
          (3000, 40, 9000, 128, 32)]
# on copies of the operands, with and without workspace; gradients in pieces; 4 bits split
COPIED = (4000, 2, 1000, 2001)
PIECES = (5000, 4, 86, 338)
SPLIT = (16, 1, 2048, 16384, 64)
# few rows of each expert in 16 bits 'T'
FEW_T = [(8, 1, 66, 1500), (16, 2, 130, 2049), (60, 20, 129, 31), (160, 20, 33, 2300), (7, 1, 65, 33000),
         (512, 64, 1030, 96)]
