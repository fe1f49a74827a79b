"""Plain float64 forms of the operators around a LookME layer, with bounds on
how far a correct float32 computation may be from them (test support).

Every function returns (value, bound).  Bounds count roundings: half a step of
the output type relative to the value, and 2^-24 of the summed magnitudes for
each float32 addition or product on the way.
"""

import torch

U32 = 2.0 ** -24                       # half a step of float32
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = 2.0 ** -126
E4M3 = torch.float8_e4m3fn


def residual_sum(hidden, add=None, part_w=None):
    s = hidden.double()
    mag = s.abs()
    parts = 0
    if add is not None:
        a = add.double()
        w = torch.ones(add.shape[:2], dtype=torch.float64) if part_w is None else part_w.double()
        parts = add.shape[1]
        a = torch.where(w[:, :, None] == 0, 0.0, a * w[:, :, None])
        s = s + a.sum(1)
        mag = mag + a.abs().sum(1)
    # a rounding a product and an addition (parts + 4 of them), each of at most
    # the magnitudes' sum
    return s, HALF[hidden.dtype] * s.abs() + (parts + 5) * U32 * (1 + 2 ** -7) * mag


def norm(stored, weight, eps):
    """y from the stored sums; the bound is float32's, without the output's
    rounding.  A thread adds at most 64 squares and the team's reduction 10
    partial sums (of positive terms: a relative error of 74 roundings, halved by
    the root; wider rows add a rounding for every 256 chunks); the mean, the
    reciprocal root (2) and the two products round 5 times more."""
    s = stored.double()
    d = s.shape[1]
    y = s / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    if weight is not None:
        y = y * weight.double()
    seq = max(64, d // 256 + 8)
    return y, ((seq + 10) / 2 + 5) * U32 * y.abs()


def silu_product(a, ea, b, eb):
    """silu(a) b with errors ea, eb in the sums: |silu'| <= 1.1; the
    exponential, the division and the products are good to 2^-20."""
    s = a / (1 + torch.exp(-a))
    v = s * b
    return v, 1.1 * ea * (b.abs() + eb) + s.abs() * eb + 2.0 ** -20 * v.abs()


def grouped(x, w, offsets, m, rows=None, picks=1, w_up=None, scatter=False, x_scale=None,
            w_scale=None, up_scale=None, out_dtype=None):
    """[m, d_out] float64 with NaN in rows that no entry writes.

    e4m3 operands: the matrix cores add the products of an aligned block of 16
    values as integers, aligned to the largest product's exponent with 13 bits
    behind its leading one, so each of the 16 loses less than 2^-13 of the
    largest product: 16 x 2^-13 = 2^-9 of it a block.  (A product 2^-13 of the
    largest counts, one 2^-14 of it does not; with the sum so far, and between
    blocks, 2^-24: a sum of 2^24 and 1.125 is 2^24 + 2.)"""
    d_in, d_out = x.shape[1], w.shape[1]
    out = torch.full((m, d_out), float("nan"), dtype=torch.float64)
    bound = torch.zeros((m, d_out), dtype=torch.float64)
    off = offsets.tolist()
    for g in range(w.shape[0]):
        i = torch.arange(off[g], off[g + 1])
        r = rows[i].long() if rows is not None else i
        src = torch.div(r, picks, rounding_mode="trunc") if rows is not None and picks else i
        dst = r if scatter else i
        ok = (r >= 0) & (src < x.shape[0]) & (dst < m)
        src, dst = src[ok], dst[ok]
        if not len(src):
            continue
        xr = x[src].double()
        both = []
        for mat, sc in ((w, w_scale), (w_up, up_scale)):
            if mat is None:
                continue
            mr = mat[g].double()
            v, e = xr @ mr.T, (d_in + 4) * U32 * (xr.abs() @ mr.abs().T)
            if x_scale is not None:
                most = lambda t: t.abs().reshape(len(t), -1, 16).amax(2)  # noqa: E731
                e = e + 2.0 ** -9 * (most(xr) @ most(mr).T)
                f = x_scale[src].double()[:, None] * sc[g].double()
                v, e = v * f, e * f + 4 * U32 * (v * f).abs()
            both.append((v, e))
        v, e = both[0] if w_up is None else silu_product(*both[0], *both[1])
        out[dst], bound[dst] = v, e + HALF[out_dtype or x.dtype] * v.abs() * (1 + 2 ** -7)
    return out, bound


def unpack(w):
    """[d_out, d_in / 2] bytes as the 4-bit values [d_out, d_in]"""
    return torch.stack([w & 15, w >> 4], 2).reshape(w.shape[0], -1)


def quant(x, w, scale, zero=None, add=None, up=None):
    """(value, bound); up: (w, scale, zero) of the second matrix.  The float32
    sums run over (16 + q) x and (16 + z) x, magnitudes of at most 31 |x| each."""
    def product(w, scale, zero):
        group = x.shape[1] // scale.shape[1]
        s = scale.double().repeat_interleave(group, 1)
        z = 8.0 if zero is None else zero.double().repeat_interleave(group, 1)
        return (x.double() @ ((unpack(w).double() - z) * s).T,
                (x.shape[1] + 8) * U32 * 62 * (x.double().abs() @ s.abs().T))
    v, e = product(w, scale, zero)
    if up is not None:
        v, e = silu_product(v, e, *product(*up))
    if add is not None:
        v = v + add.double()
        e = e + U32 * v.abs()
    return v, e + HALF[x.dtype] * v.abs() * (1 + 2 ** -7)


def pack(q):
    """4-bit values [d_out, d_in] as bytes, even columns in the low halves"""
    return (q[:, 0::2] | (q[:, 1::2] << 4)).to(torch.uint8)


def group_rows(pick, groups):
    """(entries in group order, offsets) of a stable sort"""
    lists = [[] for _ in range(groups)]
    for i, p in enumerate(pick.tolist()):
        if 0 <= p < groups:
            lists[p].append(i)
    off = [0]
    for v in lists:
        off.append(off[-1] + len(v))
    return [i for v in lists for i in v], off


def quantize_rows(v):
    """e4m3 rows with a float32 scale each"""
    scale = (v.float().abs().amax(-1) / 448).clamp_min(TINY)
    return (v.float() / scale[..., None]).to(E4M3), scale
