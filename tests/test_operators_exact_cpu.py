"""What the exact cases of the 4-bit products can see, on the CPU: a mistake in
the plain form changes what they expect."""

import pytest
import torch

from tests import operators as R
from tests import operators_exact as X


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_group_counts(dtype):
    """300 groups, more than have their scales in LDS at a time: each one's loss
    shows in every row"""
    x, w, s, z = X.quant_case(2, 9600, 16, 32, dtype, True)
    want = X.quant_sums(x, w, s, z)
    for g in range(s.shape[1]):
        t = s.clone()
        t[:, g] = 0
        assert (X.quant_sums(x, w, t, z).to(dtype) != want.to(dtype)).any(1).all(), g


@pytest.mark.parametrize("n,d_in,d_out,group", [(1, 2048, 40, 128), (16, 1120, 16, 32),
                                                (2, 9600, 16, 32), (33, 17408, 16, 128)])
def test_float32_tokens_in_fewer_bits_show(n, d_in, d_out, group):
    x, w, s, z = X.quant_case(n, d_in, d_out, group, torch.float32, False)
    less = X.quant_sums(x.to(torch.bfloat16), w, s, z)
    assert (less != X.quant_sums(x, w, s, z)).any(1).all()


def test_sums_in_float32_have_no_rounding():
    for dtype in (torch.bfloat16, torch.float32):
        x, w, s, z = X.quant_case(7, 4160, 24, 32, dtype, True)
        m = (R.unpack(w).float() - z.float().repeat_interleave(32, 1)) * \
            s.float().repeat_interleave(32, 1)
        assert torch.equal((x.float() @ m.T).double(), X.quant_sums(x, w, s, z))
