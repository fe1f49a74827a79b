"""GPU tests of every kernel of the grouped products on K of many stages, with
whole numbers whose float32 sums are exact: a stage that is dropped, taken twice
or read too early or late shows in every bit of the result."""

import pytest
import torch

from tests import grouped_plans as P
from tests import operators as R
from tests.test_gpu_operators import BF, DT, E4M3, _offsets, _say, lk  # noqa: F401

pytestmark = pytest.mark.gpu

TYPE = dict(DT, e4m3=E4M3)


def _whole(g, shape, dtype):
    """values of -7 .. 7 but 0: sums of 49 x 8192 at most, and products that a block of
    e4m3 sums keeps whole"""
    v = torch.randint(1, 8, shape, generator=g, device="cuda", dtype=torch.int8)
    v *= torch.randint(0, 2, shape, generator=g, device="cuda", dtype=torch.int8) * 2 - 1
    return v.to(dtype)


def _check(lk, name, dtype, up, k_bytes, gathered):  # noqa: F811
    more, picks = (30, 2) if gathered else (0, 0)
    sizes, d_in, d_out = P.case(name, dtype, up, k_bytes, more, picks)
    _say(name, dtype, up, sizes[:6], len(sizes), d_in, d_out, gathered)
    g = torch.Generator(device="cuda").manual_seed(21)
    dt, G, m = TYPE[dtype], len(sizes), sum(sizes) + more
    out_dt = BF if dtype == "e4m3" else dt
    x = _whole(g, (-(-m // 2) if gathered else m, d_in), dt)
    w = _whole(g, (G, d_out, d_in), dt)
    kw = {}
    if up:   # gates of a few tens (hundreds where the weights are the largest)
        w = (w.float() / 64).to(dt) if w.numel() < 2 ** 30 else w
        kw["w_up"] = _whole(g, w.shape, dt)
    if dtype == "e4m3":
        kw["x_scale"], kw["w_scale"] = (torch.ones(s, device="cuda")
                                        for s in (x.shape[:1], w.shape[:2]))
        if up:
            kw["w_up_scale"] = kw["w_scale"]
    rows = torch.randperm(m, generator=g, device="cuda").to(torch.int32) if gathered else None
    off = _offsets(sizes)
    out = torch.full((m, d_out), -9.0, dtype=out_dt, device="cuda")
    lk.grouped_product(x, w, off.cuda(), out, rows=rows, picks=picks, scatter=gathered, **kw)
    want = torch.full((m, d_out), -9.0, dtype=torch.float64, device="cuda")
    for i in range(G):
        at = torch.arange(int(off[i]), int(off[i + 1]), device="cuda")
        if not len(at):
            continue
        src = at if rows is None else rows[at].long() // picks
        dst = at if rows is None else rows[at].long()
        xs = x[src].double()
        v = xs @ w[i].double().T
        want[dst] = v if not up else v / (1 + torch.exp(-v)) * (xs @ kw["w_up"][i].double().T)
    if not up:
        assert torch.equal(out, want.to(out_dt))
        return
    # exact sums; silu and its product to 2^-20, and the output's rounding.  Below
    # -87 the exponential of float32 leaves its normal values: what is left of silu is less
    # than 128 e^-87 < 2^-118, times the other sum, below 2^19, less than 2^-99.
    bound = (2.0 ** -20 + R.HALF[out_dt] * (1 + 2 ** -7)) * want.abs() + 2.0 ** -99
    assert ((out.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("k_bytes", P.DEPTHS)
@pytest.mark.parametrize("up", [False, True])
@pytest.mark.parametrize("dtype", list(P.DT))
@pytest.mark.parametrize("name", [k for k in P.KINDS if k != "rows4 wide"])
def test_grouped_kernels_on_many_stages(lk, name, dtype, up, k_bytes):  # noqa: F811
    _check(lk, name, dtype, up, k_bytes, False)
    _check(lk, name, dtype, up, k_bytes, True)


@pytest.mark.parametrize("up", [False, True])
@pytest.mark.parametrize("dtype", list(P.DT))
def test_grouped_column_tiles_of_a_long_k(lk, dtype, up):  # noqa: F811
    """over 1 GiB of weights: several column tiles a workgroup, K over four waves"""
    _check(lk, "rows4 wide", dtype, up, P.DEPTHS[0], False)
    _check(lk, "rows4 wide", dtype, up, P.DEPTHS[0], True)
