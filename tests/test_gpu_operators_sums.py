"""GPU tests of the operators around a LookME layer on values whose float32 sums
are exact in any order: what a kernel drops, repeats or rounds on the way shows
in every bit of the result."""

import pytest
import torch

from tests import operators as R
from tests import operators_exact as X
from tests.test_gpu_operators import BF, DT, E4M3, F32, QUANT, _close, _say, lk  # noqa: F401

pytestmark = pytest.mark.gpu

# and more groups than have their scales in LDS at a time, of each kind of group
SEGMENTS = [(17, 8320, 24, 32), (1, 8256, 40, 64), (33, 17408, 16, 128), (3, 4160, 8200, 32),
            (20, 16896, 2056, 128)]


def _cuda(*ts):
    return [None if t is None else t.cuda() for t in ts]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("n,d_in,d_out,group", QUANT + SEGMENTS)
def test_quant_sums_of_whole_numbers(lk, dtype, zero, n, d_in, d_out, group):  # noqa: F811
    _say("quant exact", dtype, zero, n, d_in, d_out, group)
    x, w, s, z = X.quant_case(n, d_in, d_out, group, DT[dtype], zero)
    want = X.quant_sums(x, w, s, z)
    add = torch.randint(-1000, 1001, want.shape, generator=torch.Generator().manual_seed(9))
    add = add.to(DT[dtype])
    xd, wd, sd, zd, out = _cuda(x, w, s, z, add)
    lk.quant_product(xd, wd, sd, out, zero=zd, add=out)
    assert torch.equal(out.cpu(), (want + add.double()).to(DT[dtype]))
    lk.quant_product(xd, wd, sd, out, zero=zd)
    assert torch.equal(out.cpu(), want.to(DT[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d_in,d_out,group", QUANT + SEGMENTS)
def test_quant_swiglu_of_exact_sums(lk, dtype, n, d_in, d_out, group):  # noqa: F811
    _say("swiglu exact", dtype, n, d_in, d_out, group)
    x, w, s, z = X.quant_case(n, d_in, d_out, group, DT[dtype], True)
    _, wu, su, _ = X.quant_case(n, d_in, d_out, group, DT[dtype], False, seed=1)
    s, su = s * 2.0 ** -14, su * 2.0 ** -12
    out = torch.empty((n, d_out), dtype=DT[dtype], device="cuda")
    xd, wd, sd, zd, wud, sud = _cuda(x, w, s, z, wu, su)
    lk.quant_swiglu(xd, wd, sd, wud, sud, out, z_gate=zd)
    v, e = R.silu_product(X.quant_sums(x, w, s, z), 0.0, X.quant_sums(x, wu, su, None), 0.0)
    _close(out, v, e + R.HALF[DT[dtype]] * v.abs() * (1 + 2 ** -7), "out")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("n,group", [(1, 128), (16, 64), (3, 32), (40, 256)])
def test_quant_weights_of_zero_leave_a_value_out(lk, dtype, zero, n, group):  # noqa: F811
    """channels of huge values whose weights are q = zero: they add nothing, no
    rounding either"""
    _say("quant outliers", dtype, zero, n, group)
    d_in, d_out = 1024, 40
    x, w, s, z = X.quant_case(n, d_in, d_out, group, DT[dtype], zero)
    q = R.unpack(w)
    want = X.quant_sums(x * (torch.arange(d_in) % 100 != 77), w, s, z)
    for k, v in ((77, 3.0e38), (177, -3.0e38), (277, 1.2345678e30), (377, 54321.625)):
        x[:, k] = v
        q[:, k] = 8 if z is None else z[:, k // group]
    for k in range(477, d_in, 100):
        x[:, k] = 0
    out = torch.empty((n, d_out), dtype=DT[dtype], device="cuda")
    lk.quant_product(*_cuda(x, R.pack(q), s), out, zero=None if z is None else z.cuda())
    assert torch.equal(out.cpu(), want.to(DT[dtype]))
