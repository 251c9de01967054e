"""Which kernel the microscaled products' rule takes, and one size for every kernel that it can take."""
import ctypes

from paper_2609_24433_amd import fq


class Plan(ctypes.Structure):
    _fields_ = [("stream", ctypes.c_int), ("tile", ctypes.c_int), ("splits", ctypes.c_int), ("token", ctypes.c_bool)]


_mx_plan = fq.LIB["_ZN2fq7mx_planElll"]  # fq::mx_plan(long, long, long)
_mx_plan.argtypes = [ctypes.c_int64] * 3
_mx_plan.restype = Plan

# the rule's lists: column blocks, waves of the streaming kernels; rows, columns of the tiles
STREAM = [(1, 1, 2), (1, 1, 4), (1, 2, 4), (2, 1, 2), (2, 2, 8), (2, 4, 4), (4, 4, 4)]  # row blocks, column blocks, waves
TILE = [(64, 64), (128, 128), (128, 256), (256, 256)]


def plan(M, N, K):
    return _mx_plan(M, N, K)


def product_kind(M, N, K):
    """The kernel of a product: ("stream", shape) or ("tile", shape, whether K is split)."""
    p = plan(M, N, K)
    return ("tile", TILE[p.tile], p.splits > 1) if p.tile >= 0 else ("stream", STREAM[p.stream])


def projection_kind(M, N, K):
    """The kernel of a projection's product: the product's, or where one launch does both ("token", column blocks, waves)."""
    p = plan(M, N, K)
    if not p.token:
        return product_kind(M, N, K)
    nw = STREAM[p.stream][2]
    waves = N // 16 * nw
    return ("token", 1 if waves <= 2048 else 2 if waves <= 4096 or nw == 2 else 4, nw)


# (M, N, K) of each kernel; K ends inside a batch of four steps or inside a step of 256 channels, rows and columns inside a tile
PRODUCTS = {
    ("stream", (1, 1, 2)): (7, 1040, 640), ("stream", (1, 1, 4)): (40, 272, 1152), ("stream", (1, 2, 4)): (292, 144, 1152),
    ("stream", (2, 1, 2)): (255, 288, 384), ("stream", (2, 2, 8)): (116, 1504, 2944), ("stream", (2, 4, 4)): (694, 288, 1152),
    ("stream", (4, 4, 4)): (287, 2112, 4736),
    ("tile", (64, 64), False): (700, 2048, 384), ("tile", (64, 64), True): (1100, 80, 32640),
    ("tile", (128, 128), False): (1240, 1632, 384), ("tile", (128, 128), True): (1106, 224, 24192),
    ("tile", (128, 256), False): (1500, 4112, 896), ("tile", (128, 256), True): (866, 1200, 24192),
    ("tile", (256, 256), False): (2100, 8208, 384), ("tile", (256, 256), True): (1927, 1040, 27008),
}
# the projections of one and two tokens that take one launch; K ends inside a batch, columns inside a workgroup's
TOKENS = {("token", 1, 2): (2, 144, 640), ("token", 2, 2): (2, 20496, 384), ("token", 1, 4): (1, 272, 1152),
          ("token", 2, 4): (1, 12304, 1152), ("token", 4, 4): (2, 20496, 1152)}
