"""GPU tests of the operators around a LookME layer on values whose float32 sums
are exact in any order: what a kernel drops, repeats or rounds on the way shows
in every bit of the result."""

import pytest
import torch

from tests import operators as R
from tests import operators_exact as X
from tests.test_gpu_operators import BF, DT, E4M3, KERNELS, QUANT, _close, _offsets, _say, lk  # noqa: F401

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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d_out", [(2 ** 20 - 16, 8), (3, 2 ** 21 + 8), (40, 2 ** 18)])
def test_quant_products_of_the_most_rows_and_columns(lk, dtype, n, d_out):  # noqa: F811
    _say("quant large", dtype, n, d_out)
    x, w, s, z = X.quant_case(16, 64, 4096, 32, DT[dtype], True)
    xs, ws = x.repeat(-(-n // 16), 1)[:n], w.repeat(-(-d_out // 4096), 1)[:d_out]
    ss, zs = (t.repeat(-(-d_out // 4096), 1)[:d_out] for t in (s, z))
    out = torch.empty((n, d_out), dtype=DT[dtype], device="cuda")
    lk.quant_product(*_cuda(xs, ws, ss), out, zero=zs.cuda())
    want = X.quant_sums(x, w, s, z).to(DT[dtype]).cuda()
    for a in range(0, n, 16):
        if n <= 64 or a % 65536 == 0 or a + 16 >= n:
            for b in range(0, d_out, 4096):
                got = out[a:a + 16, b:b + 4096]
                assert torch.equal(got, want[:got.shape[0], :got.shape[1]]), (a, b)
    full = out[:n // 16 * 16]
    if d_out < 4096:
        assert (full.view(-1, 16, d_out) == want[:, :d_out]).all()


# ---------------------------------------------------------------------------
# e4m3 grouped products
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("up", [False, True])
@pytest.mark.parametrize("sizes,d_in,d_out", KERNELS)
def test_grouped_scales_whose_product_has_no_float32(lk, sizes, d_in, d_out, up):  # noqa: F811
    """rows and columns of very large and very small scales: a sum of zero stays
    zero, a small result keeps its digits.  Up to two values of a row are not 0, so the sums
    are exact; two roundings of the scaled sum and one of the output"""
    _say("grouped scales", sizes[:8], d_in, d_out, up)
    g = torch.Generator().manual_seed(11)
    G, m = len(sizes), sum(sizes)
    x = torch.zeros((m, d_in))
    for _ in range(2):
        x[torch.arange(m), torch.randint(0, d_in, (m,), generator=g)] = \
            2.0 ** torch.randint(-3, 9, (m,), generator=g)
    w = torch.randint(1, 16, (G, d_out, d_in), generator=g).float()
    kind = torch.arange(m) % 4        # sums of zero, small, large, and ordinary
    x[kind == 0] = 0
    xs = (1 + torch.rand((m,), generator=g)) * torch.tensor([2.0 ** 100, 2.0 ** -70, 2.0 ** 70, 1.0])[kind]
    of = torch.arange(d_out) % 3
    ws = (1 + torch.rand((G, d_out), generator=g)) * torch.tensor([2.0 ** 40, 2.0 ** -72, 1.0])[of]
    out = torch.full((m, d_out), -7.0, dtype=BF, device="cuda")
    off = _offsets(sizes)
    kw = dict(w_up=w.to(E4M3).cuda(), w_up_scale=torch.ones((G, d_out), device="cuda")) if up else {}
    lk.grouped_product(x.to(E4M3).cuda(), w.to(E4M3).cuda(), off.cuda(), out, x_scale=xs.cuda(),
                       w_scale=ws.cuda(), **kw)
    got, inside = out.cpu(), 0
    assert (got[kind == 0] == 0).all(), "sums of zero"
    for i in range(G):
        a, b = int(off[i]), int(off[i + 1])
        s = x[a:b].double() @ w[i].double().T
        v = s * xs[a:b, None].double() * ws[i].double()
        e = 3 * R.U32 * v.abs()
        if up:
            u = s * xs[a:b, None].double()
            v, e = R.silu_product(v, e, u, 2 * R.U32 * u.abs())
        # (bf16's numbers end at 2^128, its steps at 2^-133)
        e = e + R.HALF[BF] * v.abs() * (1 + 2 ** -7) + 2.0 ** -134
        fits = v.abs() < 2.0 ** 127
        inside += int(fits.sum())
        r = got[a:b].double()
        assert (((r - v).abs() <= e) | ~fits).all(), f"group {i}"
    assert inside >= 0.7 * got.numel()   # (but most of one row in four)


@pytest.mark.parametrize("sizes,d_in,d_out", KERNELS)
def test_grouped_e4m3_blocks_of_eight(lk, sizes, d_in, d_out):  # noqa: F811
    """products of 2^16 and -2^16 in two blocks of 8 neighbouring values, and one of 1 in a third
    or one of 8 beside the first: both are there in every kernel"""
    _say("grouped blocks", sizes[:8], d_in, d_out)
    g = torch.Generator().manual_seed(12)
    m, G = sum(sizes), len(sizes)
    block = torch.stack([torch.randperm(d_in // 8, generator=g)[:3] for _ in range(m)]) * 8
    at = block + torch.randint(0, 8, (m, 3), generator=g)
    beside = block[:, 0] + (at[:, 0] % 8 + 1 + torch.randint(0, 7, (m,), generator=g)) % 8
    i, third = torch.arange(m), torch.arange(m) % 2 == 0
    x = torch.zeros((m, d_in))
    x[i, at[:, 0]], x[i, at[:, 1]] = 256.0, -256.0
    x[i, at[:, 2]] = torch.where(third, 1.0 / 256, 0.0)     # an e4m3 value, of weight 256: 1
    x[i, beside] = torch.where(third, 0.0, 1.0 / 32)        # 8 = 2^-13 of 2^16
    out = torch.empty((m, d_out), dtype=BF, device="cuda")
    w = torch.full((G, d_out, d_in), 256.0).to(E4M3)
    lk.grouped_product(x.to(E4M3).cuda(), w.cuda(), _offsets(sizes).cuda(), out,
                       x_scale=torch.ones(m, device="cuda"),
                       w_scale=torch.ones((G, d_out), device="cuda"))
    want = torch.where(third, 1.0, 8.0)[:, None].expand(m, d_out)
    assert torch.equal(out.cpu().float(), want)
