"""Plain float64 forms of the operators of an attention sublayer, with bounds on
how far a correct float32 computation may be from them (test support).

Every function with a bound returns (value, bound).  Bounds count roundings: half a
step of the output type relative to the value, and 2^-24 of the summed magnitudes
for each float32 addition or product on the way.
"""

import math

import torch

U32 = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


# ---- the cache -----------------------------------------------------------------

def quantize(x):
    """x [..., d] as (codes [..., d], scale bytes [..., d / 32])"""
    x = x.double()
    blocks = x.unflatten(-1, (-1, 32))
    top = blocks.abs().amax(-1)
    finite = torch.isfinite(blocks).all(-1)
    top = torch.where(finite, top, 1.0)
    exponent = torch.full(top.shape, -100, dtype=torch.int64)
    for e in range(-100, 125):       # the smallest of them that holds the block
        exponent = torch.where(top > 7 * 2.0 ** e, e + 1, exponent)
    unit = torch.pow(torch.tensor(2.0, dtype=torch.float64), exponent.double())
    far = (blocks.abs()[..., None] / unit[..., None, None] - GRID).abs()
    far = torch.where(torch.isfinite(far), far, 0.0)
    near = far.amin(-1, keepdim=True)
    # of two as near, the even code
    code = torch.where(far == near, torch.arange(8) % 2 * 8 + torch.arange(8), 99).amin(-1) % 8
    code = torch.where(finite[..., None], code + 8 * torch.signbit(blocks), 0)
    byte = torch.where(finite, exponent + 127, 255)
    return code.flatten(-2).to(torch.uint8), byte.to(torch.uint8)


def value(code, byte):
    """The values of codes [..., d] with scale bytes [..., d / 32]"""
    v = GRID[(code & 7).long()] * torch.where(code >= 8, -1.0, 1.0)
    s = torch.pow(torch.tensor(2.0, dtype=torch.float64), byte.double() - 127)
    s = torch.where(byte == 255, math.nan, s)
    return (v.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def places(t, d):
    """Bytes in a tile of token t: k and v codes of the even dims, k and v scales"""
    k, v, u = [], [], d // 16
    for dim in range(0, d, 2):
        k.append(t * d // 2 + dim % 32 // 8 * (d // 8) + dim // 32 * 4 + dim % 8 // 2)
        v.append(16 * d + ((t % 16 // 4 * 16 + dim // u) * 8 + t % 4 + 4 * (t // 16)) * (u // 2)
                 + dim % u // 2)
    g = range(d // 32)
    return (torch.tensor(k), torch.tensor(v), torch.tensor([32 * d + t * (d // 32) + i for i in g]),
            torch.tensor([33 * d + i * 32 + t % 16 // 4 * 8 + t % 4 + 4 * (t // 16) for i in g]))


def write(cache, slots, k, v):
    """cache [pages, heads, page / 32, 34 d] with the rows in their slots (a new tensor)"""
    cache = cache.clone()
    pages, heads, tiles, width = cache.shape
    d, page = width // 34, tiles * 32
    where = [places(t, d) for t in range(32)]
    (kc, ks), (vc, vs) = quantize(k), quantize(v)
    pack = lambda c: c[..., 0::2] | (c[..., 1::2] << 4)  # noqa: E731
    kc, vc = pack(kc), pack(vc)
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < pages * page:
            at = cache[s // page, :, s % page // 32]
            for p, x in zip(where[s % 32], (kc[i], vc[i], ks[i], vs[i])):
                at[:, p] = x
    return cache


def read(cache, slots):
    """float64 (k, v) [n, heads, d] of slots that are all in range"""
    pages, heads, tiles, width = cache.shape
    d, page = width // 34, tiles * 32
    where = [places(t, d) for t in range(32)]
    s = torch.as_tensor(slots).long()
    rows = cache[s // page, :, s % page // 32]                          # [n, heads, 34 d]
    out = []
    for a, b in ((0, 2), (1, 3)):
        at = torch.stack([where[i][a] for i in (s % 32).tolist()]) if len(s) else torch.empty(
            (0, d // 2), dtype=torch.long)
        sc = torch.stack([where[i][b] for i in (s % 32).tolist()]) if len(s) else torch.empty(
            (0, d // 32), dtype=torch.long)
        codes = torch.gather(rows, 2, at[:, None].expand(-1, heads, -1))
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
        out.append(value(codes, torch.gather(rows, 2, sc[:, None].expand(-1, heads, -1))))
    return out


# ---- head norms and positions --------------------------------------------------

def rotary(x, weight=None, eps=None, pos=None, freq=None, axis=None, factor=1.0,
           interleaved=False):
    """x [n, heads, d]; eps None: no norm.  The norm's float32 sums add at most 8
    values a lane and 6 partial sums of positive terms, halved by the root; mean,
    root (2) and products round 6 times more.  An angle in turns, at most half a
    turn, is good to 2^-26 + 2^-51 of the whole turns, so 2 pi times that; sine and
    cosine to 2^-22 more; their products and the sum round 4 times."""
    y = x.double()
    n, d = x.shape[0], x.shape[2]
    e = torch.zeros_like(y)
    if eps is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
        if weight is not None:
            y = y * weight.double()
        e = (7 + 6 + 2) * U32 * y.abs()
    if freq is not None:
        half = freq.numel()
        pos = pos.double().reshape(-1, n)
        pos = pos[axis.long()] if axis is not None else pos[:1].expand(half, n)
        turns = pos.T * freq.double() / (2 * math.pi)
        angle = 2 * math.pi * (turns - turns.round())
        c, s = torch.cos(angle)[:, None] * factor, torch.sin(angle)[:, None] * factor
        ea = (2 * math.pi * (2.0 ** -26 + 2.0 ** -51 * turns.abs())[:, None] + 2.0 ** -22
              + U32) * abs(factor)
        i = torch.arange(half)
        i0, i1 = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        z, ez = y.clone(), e.clone()
        a, b, xa, xb = y[..., i0], y[..., i1], e[..., i0], e[..., i1]
        both = a.abs() + b.abs()
        z[..., i0], z[..., i1] = a * c - b * s, a * s + b * c
        more = (ea + 4 * U32 * abs(factor)) * both + (xa + xb) * abs(factor) * (1 + 2.0 ** -20)
        ez[..., i0] = ez[..., i1] = more
        y, e = z, ez
    return y, e + HALF[x.dtype] * y.abs() * (1 + 2.0 ** -7) + 2.0 ** -126


# ---- attention -------------------------------------------------------------------

def attention(q, k, v, scale, causal):
    """One sequence: q [m, q_heads, d], k and v [n, kv_heads, d] float64.

    A score adds d products (three parts a float32 query, whose bits they hold): (d +
    16) 2^-24 of the magnitudes' sum.  The exponent is a float32 of the scaled score
    less the maximum's, each good to 2^-23 of the largest |score log2 e|, the exponential to
    2^-22; an error of x in a score is one of x in its weight, and at most as much
    in their sum.  Weights and outputs are sums over n: (n + 64) 2^-24, and bf16
    weights round once, 2^-8."""
    m, hq, d = q.shape
    n, hkv = k.shape[:2]
    out = torch.zeros((m, hq, d), dtype=torch.float64)
    bound = torch.zeros_like(out)
    seen = torch.full((m,), n) if not causal else torch.arange(m) + n - m + 1
    for h in range(hq):
        kh, vh = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)]
        qh = q[:, h].double()
        for i in range(m):
            t = int(seen[i])
            if t <= 0:
                continue
            s = scale * (kh[:t] @ qh[i])
            mag = scale * (kh[:t].abs() @ qh[i].abs())
            p = torch.softmax(s, 0)
            out[i, h] = p @ vh[:t]
            x = (d + 16) * U32 * mag.max() + 4 * U32 * (1.5 * s.abs().max() + 16) + 2.0 ** -21
            part = 2 * x + (t + 64) * U32
            if q.dtype == torch.bfloat16:
                part = part + HALF[q.dtype] * (1 + 2.0 ** -7)
            bound[i, h] = part * (p @ vh[:t].abs())
    return out, bound + HALF[q.dtype] * out.abs() * (1 + 2.0 ** -7) + 2.0 ** -126
