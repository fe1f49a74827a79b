"""Support of the tests of attention's kernel of many rows: the rule that chooses it,
called in the built library (host code), calls that it chooses it for, and a float64 form
of all rows at once."""

import ctypes

import torch

from paper_2607_16305_amd import lookme as lk
from tests import attention as A

DT = {"f32": lk.LOOKME_F32, "bf16": lk.LOOKME_BF16}


class Plan(ctypes.Structure):
    _fields_ = [("tiles", ctypes.c_int), ("block", ctypes.c_int), ("target", ctypes.c_int),
                ("units", ctypes.c_int64), ("tile_us", ctypes.c_float),
                ("join_us", ctypes.c_float)]


def plan(dtype, n, batch, q_heads, kv_heads, d, tokens):
    """tokens: what the page table of a sequence could hold"""
    f = lk.load()._ZN6lookme11attend_planEiliiiil
    f.argtypes = [ctypes.c_int, ctypes.c_int64] + [ctypes.c_int] * 4 + [ctypes.c_int64]
    f.restype = Plan
    return f(DT[dtype], n, batch, q_heads, kv_heads, d, tokens)


# the kernel of many rows (its waves along the rows) is built for these
MANY = [("bf16", 128), ("bf16", 256), ("f32", 128)]
PAGE = 32


def _spread(batch, rows, length):
    """(rows, length) of sequences about as long, with a short one and ones without rows or
    tokens"""
    seqs = [(rows + i % 5 - 2, length - 7 * i % 60) for i in range(batch)]
    seqs[3], seqs[5], seqs[7], seqs[-1] = (9, 0), (0, 40), (rows, 1), (5, 3)
    return seqs


# (sequences, q heads, key heads, pages of a table, whether the host leaves the keys whole).
# Without a cut the rows fill most of the chip; more than 64 sequences are searched.
CALLS = {
    "whole": (_spread(25, 40, 250), 30, 6, 8, True),
    "whole, many sequences": (_spread(80, 15, 90), 20, 2, 3, True),
    "whole, decode rows beside a prompt": ([(1, 20 * i + 1) for i in range(6)] + [(600, 600)] +
                                           [(1, 40 * i + 300) for i in range(6)], 32, 4, 20, True),
    "whole, as the kernel finds": ([(300, 320), (290, 290)], 16, 2, 2000, False),
    "cut": ([(50, 700), (37, 222), (60, 64), (45, 20), (0, 90)], 12, 3, 80, False),
    "cut, many sequences": (_spread(70, 14, 60)[:-1] + [(20, 2300)], 8, 1, 75, False),
}


def of(name, dtype, d):
    seqs, hq, hkv, width, _ = CALLS[name]
    return plan(dtype, sum(m for m, _ in seqs), len(seqs), hq, hkv, d, width * PAGE)


def attention(q, k, v, scale, causal, keep=None):
    """attention.attention of all rows at once, with its bound; keep [n]: tokens that are on
    some page.

    The bound holds what float32 loses at its lower end too: weights are relative to a
    maximum, up to 2^8, and add up to at least 1; what is below 2^-126 of them may be
    flushed as a weight (three parts of a float32 one), where waves are joined, and where
    parts of the keys are: (2 2^8 + 3) 2^-126, below 2^-116, of the sum of |v|."""
    m, hq, d = q.shape
    n, hkv = k.shape[:2]
    G = hq // hkv
    if m == 0 or n == 0:
        zero = torch.zeros((m, hq, d), dtype=torch.float64)
        return zero, zero + 2.0 ** -126
    qh = q.double().view(m, hkv, G, d).permute(1, 0, 2, 3).reshape(hkv, m * G, d)
    kh, vh = k.permute(1, 2, 0).contiguous(), v.permute(1, 0, 2).contiguous()
    last = torch.arange(m) + n - m if causal else torch.full((m,), n - 1)
    seen = torch.arange(n) <= last[:, None]
    if keep is not None:
        seen = seen & keep
    seen = seen.repeat_interleave(G, 0)                                # [m G, n]
    s = scale * torch.bmm(qh, kh)
    mag = (scale * torch.bmm(qh.abs(), kh.abs())).masked_fill(~seen, 0).amax(-1, keepdim=True)
    top = s.abs().masked_fill(~seen, 0).amax(-1, keepdim=True)
    p = torch.softmax(s.masked_fill(~seen, -torch.inf), -1)
    p = p.masked_fill(~seen, 0)                                        # (rows that see nothing)
    out, size = torch.bmm(p, vh), torch.bmm(p, vh.abs())
    x = (d + 16) * A.U32 * mag + 4 * A.U32 * (1.5 * top + 16) + 2.0 ** -21
    part = 2 * x + (seen.sum(-1)[:, None] + 64) * A.U32
    if q.dtype == torch.bfloat16:
        part = part + A.HALF[q.dtype] * (1 + 2.0 ** -7)
    size_all = vh.abs().sum(1, keepdim=True)
    bound = (part * size + 2.0 ** -116 * size_all +
             A.HALF[q.dtype] * out.abs() * (1 + 2.0 ** -7) + 2.0 ** -126)
    back = lambda t: t.view(hkv, m, G, d).permute(1, 0, 2, 3).reshape(m, hq, d)  # noqa: E731
    return back(out), back(bound)
