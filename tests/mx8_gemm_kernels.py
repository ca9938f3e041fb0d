"""Sizes of products of 8-bit activations and 4-bit weights at which each of their kernels runs: one group and several,
with SwiGLU and without, an odd and an even number of steps of 128 values, more tiles than workgroups stay for, and last
tiles of every number of rows."""
import ctypes

from paper_2608_07814_amd import lorex as lx

KERNELS = ("rows", "rows4", "tile64", "tile128", "tile256")
TILE = {"rows": (16, 64), "rows4": (16, 32), "tile64": (64, 128), "tile128": (128, 128), "tile256": (256, 256)}
AT_ONCE = {"tile64": 512, "tile128": 512, "tile256": 256}  # workgroups of a launch

# (kernel, SwiGLU, M, N, K, groups)
CASES = [
    ("rows4", False, 37, 104, 1160, 1), ("rows4", True, 19, 208, 640, 1), ("rows4", False, 150, 104, 640, 9), ("rows4", True, 90, 144, 1160, 5),
    ("rows", False, 61, 1032, 640, 20), ("rows", True, 300, 528, 1032, 100),
    ("tile64", False, 8265, 912, 640, 1), ("tile64", True, 1665, 4688, 136, 1), ("tile64", False, 1165, 3384, 1160, 20), ("tile64", True, 1165, 3392, 640, 20),
    ("tile128", False, 8965, 1304, 640, 1), ("tile128", True, 8265, 1824, 1160, 1), ("tile128", False, 5965, 1304, 1032, 20), ("tile128", True, 2065, 4688, 640, 20),
    ("tile256", False, 20851, 1320, 2312, 1), ("tile256", True, 22042, 1056, 640, 1), ("tile256", False, 16200, 2312, 2312, 20), ("tile256", True, 2192, 7920, 1160, 7),
]


def kernel(M, N, K, G, swiglu, rows_only=False):
    """The kernel that the library chooses (its lx::mx8_gemm_plan)."""
    f = lx.lib()._ZN2lx13mx8_gemm_planEiiiibb
    f.restype, f.argtypes = ctypes.c_int32, [ctypes.c_int32] * 4 + [ctypes.c_bool] * 2
    return KERNELS[f(M, N, -(-K // 128) * 128, G, swiglu, rows_only)]
