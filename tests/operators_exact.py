"""Inputs of the 4-bit products whose sums are whole numbers below 2^24 in any
order, so that a float32 computation has no rounding at all (test support)."""

import torch

from tests import operators as R


def quant_case(n, d_in, d_out, group, dtype, zero, seed=0):
    """(x, w, scale, zero): every |x| is at most `most`, but in one column of 128
    (float32 only) up to 2047, which takes more bits than a bf16 value has;
    weights at most 15, scales 1 or 2: sums of at most
    30 (most d_in + 2047 (d_in / 128 + 1)) < 2^24."""
    g = torch.Generator().manual_seed(1000 * seed + n + d_in + d_out + group)
    most = min(100, 2 ** 23 // (30 * d_in))
    x = torch.randint(-most, most + 1, (n, d_in), generator=g).float()
    x = torch.where(x == 0, 1.0, x)
    if dtype is torch.float32:
        for k in range(0, d_in, 128):
            at = k + int(torch.randint(0, min(128, d_in - k), (1,), generator=g))
            x[:, at] = torch.randint(1024, 2048, (n,), generator=g).float()
    assert 30 * float(x.abs().sum(1).max()) < 2 ** 24
    w = torch.randint(0, 256, (d_out, d_in // 2), generator=g, dtype=torch.uint8)
    s = torch.randint(1, 3, (d_out, d_in // group), generator=g).to(dtype)
    z = torch.randint(0, 16, s.shape, generator=g, dtype=torch.uint8) if zero else None
    return x.to(dtype), w, s, z


def quant_sums(x, w, scale, zero):
    """sum_G scale_G sum_{k in G} (q_k - zero_G) x_k in 64 bits"""
    group = x.shape[1] // scale.shape[1]
    z = 8.0 if zero is None else zero.double().repeat_interleave(group, 1)
    m = (R.unpack(w).double() - z) * scale.double().repeat_interleave(group, 1)
    return x.double() @ m.T
