"""Which kernels make a product with an epilogue, as the library's own choice says, and sizes beside those of fp8_plans.py that the choice needs."""
import ctypes

import paper_2104_07857_amd as zi

Y8, TURNED, BOTH = zi.ZI_EPILOGUE_Y8, zi.ZI_EPILOGUE_TURNED, zi.ZI_EPILOGUE_Y8 | zi.ZI_EPILOGUE_TURNED


class Plan(ctypes.Structure):
    _fields_ = [("shape", ctypes.c_int), ("parts", ctypes.c_uint32), ("part_steps", ctypes.c_uint32), ("whole", ctypes.c_int32)]


def plan(m, n, k, outputs8):
    f = ctypes.CDLL(zi.LIB_PATH)._ZN2zi24plan_fp8_matmul_epilogueEllli
    f.restype, f.argtypes = Plan, [ctypes.c_int64] * 3 + [ctypes.c_int]
    return f(m, n, k, outputs8)


# sums of tiles of 64 x 128, of which a second kernel makes the transposed numbers
SUMS = [(320, 6050, 8001), (300, 5003, 6100)]
# outputs in 8 bits from tiles of 256 x 256 and of 256 x 128
ALONE = [(1550, 7587, 4143), (3087, 1283, 9049)]
