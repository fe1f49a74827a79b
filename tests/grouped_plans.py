"""The rule that chooses a grouped product's kernel, called in the built library
(host code), and sizes for each of its choices (test support)."""

import ctypes

from paper_2607_16305_amd import lookme as lk

DT = {"f32": 0, "bf16": 1, "e4m3": 2}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}
ROWS, RING, TILES = 0, 1, 2


class Plan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("kernel", "depth", "rows", "span", "blocks")]


def plan(dtype, up, sizes, d_in, d_out, picks=0, x_rows=None, m=None):
    """sizes: the groups' rows (their number and sum count)"""
    f = lk.load()._ZN6lookme12grouped_planEibliilil
    f.argtypes = [ctypes.c_int, ctypes.c_bool, ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                  ctypes.c_int64, ctypes.c_int, ctypes.c_int64]
    f.restype = Plan
    m = sum(sizes) if m is None else m
    return f(DT[dtype], up, m, len(sizes), d_out, d_in * BYTES[dtype], picks,
             m if x_rows is None else x_rows)


# every kernel that a launch can take: (kernel, K's waves or the ring's stages, rows of
# a tile, whether a workgroup takes several column tiles)
KINDS = {"rows2": (ROWS, 2, 16, False), "rows4": (ROWS, 4, 16, False),
         "rows2 wide": (ROWS, 2, 16, True), "rows4 wide": (ROWS, 4, 16, True),
         "ring3 32": (RING, 3, 32, False), "ring4 32": (RING, 4, 32, False),
         "ring2 64": (RING, 2, 64, False), "ring4 64": (RING, 4, 64, False),
         "tiles": (TILES, 0, 0, False)}
# K in bytes: stages of 128 and a tail of 16-byte chunks, an odd and an even number of
# stages, and whole ones
DEPTHS = [1200, 1296, 1408]
CANDIDATES = [([1] * 64, 512), ([3, 0, 2, 1], 72), ([1, 2, 0, 1] * 375, 520), ([1] * 128, 1040),
              ([20] * 64, 1024), ([20, 31, 9, 0] * 8, 512), ([70, 65, 75] * 11, 1024),
              ([70, 65, 75] * 5, 1024), ([70, 65, 75] * 5, 512), ([64, 3, 160, 120] * 24, 1024),
              ([1500, 0, 2000, 300, 1, 130] + [46] * 18, 4096), ([1, 0, 2, 1] * 4, 72),
              ([2471, 2500, 2443, 2400, 2506, 2506], 1824)]


def kind(p):
    for name, k in KINDS.items():
        if (p.kernel, p.depth, p.rows, p.span > 1) == k:
            return name
    return None


def case(name, dtype, up, k_bytes, m_more=0, picks=0):
    """(sizes, d_in, d_out) that the rule sends to kernel `name`; K of at least
    8 KiB where only that leads there"""
    if name == "rows4 wide":
        k_bytes += 7168
    d_in = k_bytes // BYTES[dtype]
    for sizes, d_out in CANDIDATES:
        m = sum(sizes) + m_more
        x_rows = -(-m // picks) if picks else m
        if kind(plan(dtype, up, sizes, d_in, d_out, picks, x_rows, m)) == name:
            return sizes, d_in, d_out
    return None
