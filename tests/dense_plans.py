"""Which kernels and tiles the sizes of the dense products' tests come to (csrc/spdnn_linear_plan.h, through its host build), and sizes for
those that need many rows or columns.

A name is the tile, 64, 128 or 256, with the number of stages in LDS behind a dot (one workgroup to a CU has three), or few1, few2, few4 for
the kernel for few rows (n: tiles of 16 columns), and "/s" where k is in parts."""
import ctypes

from paper_2007_14152_amd import build as hip_build


def _lib():
    L = ctypes.CDLL(hip_build.ORDER_HOST_LIB)
    i32, out = ctypes.c_int, ctypes.c_int64 * 8
    L.spdnn_linear_plan_host.argtypes = [i32] * 8 + [out]
    L.spdnn_weight_grad_plan_host.argtypes = [i32] * 6 + [out]
    return L, out()


def _name(p):
    few, narrow, tile, _, alone, splits = p[:6]
    name = "few%d%s" % (few, "n" if narrow else "") if few else "256" if tile == 256 else "%d.%d" % (tile, 3 if alone else 2)
    return name + ("/s" if splits > 1 else "")


def product(rows, k, cols, experts, float32, k_adjacent):
    """experts: None for one matrix.  x of rows x k; W of k x cols, its k adjacent in memory or its columns."""
    L, out = _lib()
    L.spdnn_linear_plan_host(rows, k, cols, experts is not None, experts or 1, 0 if float32 else 1, 1, k_adjacent, out)
    return _name(out)


def weight_grad(rows, m, n, experts, float32):
    """W stored as m rows of n."""
    L, out = _lib()
    L.spdnn_weight_grad_plan_host(rows, m, n, experts or 1, 0 if float32 else 1, 1, out)
    return _name(out)


# (name, rows, k, cols): x W and, with the batch as k, its gradient
PRODUCTS_16 = [("64.3", 131, 41, 35), ("64.3/s", 131, 4101, 35), ("64.2", 8201, 41, 67), ("64.2/s", 259, 8201, 67), ("128.2", 2051, 41, 2053),
               ("128.2", 4099, 200, 1100), ("128.2/s", 8201, 8201, 67), ("128.3", 903, 6003, 4001), ("256", 2051, 41, 4103), ("256", 2051, 333, 4103),
               ("256", 2304, 320, 4096), ("256/s", 131, 8201, 6001)]
PRODUCTS_32 = [("64.2", 131, 41, 35), ("64.2/s", 259, 8201, 67), ("128.2", 901, 131, 8001), ("128.2", 1024, 128, 8192), ("128.2/s", 901, 8201, 901),
               ("256", 1001, 131, 16001), ("256", 1024, 160, 16000)]
GRADS_16 = [("64.3", 41, 35, 35), ("64.3/s", 4101, 35, 35), ("64.2", 41, 67, 8201), ("64.2/s", 8201, 131, 131), ("128.2", 41, 2051, 2053),
            ("128.2", 333, 1100, 4099), ("128.2/s", 8201, 67, 8201), ("128.3", 6001, 903, 4001), ("256", 41, 2051, 4103), ("256", 333, 2051, 4103),
            ("256", 320, 2304, 4096), ("256/s", 8201, 131, 6001)]
GRADS_32 = [("64.2", 41, 35, 35), ("64.2/s", 777, 35, 35), ("128.2", 131, 901, 8001), ("128.2/s", 8201, 901, 901), ("256", 131, 1001, 16001),
            ("256", 160, 1024, 16000)]
# (name, loads, k, cols): rows of the experts, and of none behind them
GROUPED_16 = [("64.3", (100, 0, 57, 64), 5, 41, 35), ("64.3/s", (100, 0, 57, 64), 5, 4101, 35), ("64.2", (3000, 0, 2001, 3200), 1, 41, 67),
              ("64.2/s", (90, 64, 65, 1, 0, 129, 63, 60, 70, 80, 75, 60), 9, 4101, 35),
              ("128.2", (90, 64, 65, 1, 0, 129, 63, 60, 70, 80, 75, 60), 9, 41, 3001), ("128.2/s", (2000, 513, 0, 3480), 9, 8201, 67),
              ("128.3", (300, 1, 0, 200, 499), 3, 6001, 2501),
              # experts that end with the first row of a tile, in its first half, with it, in its second half, and with the last
              ("256", (257, 0, 128, 640, 129, 385, 512, 200), 5, 200, 3331), ("256", (257, 0, 128, 640, 129, 385, 512, 200), 0, 128, 3328),
              ("256/s", (2500, 0, 3490), 11, 8201, 131)]
GROUPED_32 = [("64.2", (100, 0, 57, 64), 5, 41, 35), ("64.2/s", (90, 0, 65), 4, 777, 35), ("128.2", (4000, 0, 3901), 10, 131, 901),
              ("128.2/s", (1001, 898), 1, 6001, 901), ("256", (7600, 1, 8000), 10, 131, 1001)]
# (name, loads, dropped, m, n): gradients of the experts' matrices
GROUPED_GRADS_16 = [("64.3", (20, 0, 21), 3, 35, 35), ("64.3/s", (2000, 0, 2101), 3, 35, 35), ("64.2", (3, 1, 0, 4, 9, 5, 2, 8, 3, 3, 3, 1), 2, 35, 1501),
                    ("64.2/s", (2000, 0, 2101), 3, 35, 1501), ("128.2", (3, 1, 0, 4, 9, 5, 2, 8, 3, 3, 3, 1), 2, 779, 2051),
                    ("128.2", (257, 64, 65, 1, 0, 129, 63, 60, 70, 80, 75, 60), 2, 779, 2051),
                    ("256", (3, 1, 0, 4, 9, 5, 2, 8, 3, 3, 3, 1), 2, 1501, 1503), ("256", (257, 64, 65, 1, 0, 129, 63, 60, 70, 80, 75, 60), 2, 1501, 1503)]
GROUPED_GRADS_32 = [("64.2", (20, 0, 21), 3, 35, 35), ("64.2/s", (400, 0, 377), 3, 35, 35), ("128.2", (70, 61), 3, 1001, 12001),
                    ("128.2/s", (6001, 6000), 3, 251, 12001), ("256", (71, 60), 2, 2001, 12003)]
# few rows, whose rule depends on the type and on how W is stored: (rows, k, cols), (loads, dropped, k, cols)
FEW = [(rows, k, cols) for rows in (3, 29, 100) for k, cols in ((41, 37), (1001, 131), (8201, 67), (41, 16391))]
FEW_GROUPED = [(loads, 3, k, cols) for loads in ((1, 0, 3, 7), (9, 20, 0, 12), (40, 0, 33, 9)) for k, cols in ((41, 37), (4101, 37), (333, 6001))]
