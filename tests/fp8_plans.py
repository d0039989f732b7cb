"""Which kernel makes a product in 8 bits, as the library's own choice says, and sizes of which each kernel has some."""
import ctypes

import paper_2104_07857_amd as zi

SHAPES = [(64, 64), (64, 128), (128, 128), (128, 128), (256, 128), (256, 256)]     # rows and columns of tiles
FEW = -1


class Plan(ctypes.Structure):
    _fields_ = [("shape", ctypes.c_int), ("parts", ctypes.c_uint32), ("part_steps", ctypes.c_uint32)]


def plan(m, n, k):
    f = ctypes.CDLL(zi.LIB_PATH)._ZN2zi15plan_fp8_matmulElll
    f.restype, f.argtypes = Plan, [ctypes.c_int64] * 3
    return f(m, n, k)


# up to 16 rows of A: the second and later turns of a workgroup's k (4096 each), a last run (of 512) that is short, one block and less of it
FEW_16 = [(1, 5000, 20001), (4, 2048, 16384), (8, 1024, 16300), (12, 257, 9001), (16, 100, 4097), (9, 33, 4096 + 512 + 384), (16, 15, 130)]
# 17 to 32
FEW_32 = [(20, 300, 2000), (32, 1024, 4000), (25, 1000, 4097), (17, 100, 8192), (32, 333, 4700), (31, 47, 4096 + 512 + 256), (18, 16, 1000)]
# parts of k: last parts and blocks that are short, columns beyond a workgroup of the sum over parts and that end inside four
PARTS = [(40, 200, 16384), (33, 129, 12345), (300, 40, 3000), (100, 64, 7000), (64, 1500, 8000), (200, 1026, 9000), (24, 1031, 12001), (16, 8192, 8000)]
# the six tiles: ends on all sides, k that ends inside a block, inside a group of four blocks, with a group
TILES = [(33, 128, 256), (65, 70, 512), (129, 255, 513), (300, 520, 640), (257, 511, 1030), (17, 8192, 1111),
         (1290, 3000, 384), (1290, 3001, 1667), (1290, 1545, 4001), (2049, 1001, 4001), (2500, 1544, 200), (2049, 2047, 1000), (1001, 4099, 4001),
         (2049, 2047, 4001), (1290, 3500, 4224), (2049, 6001, 1667), (3001, 4099, 2560), (3001, 4100, 3000)]
