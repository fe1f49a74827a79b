"""GPU tests of grouped products whose operands pass 2 and 4 GiB, in every kernel
that addresses them, with whole numbers whose float32 sums are exact."""

import pytest
import torch

from tests import grouped_plans as P
from tests.test_gpu_operators import BF, E4M3, _say, lk  # noqa: F401
from tests.test_gpu_operators_depth import TYPE, _whole

pytestmark = pytest.mark.gpu

GIB = 1 << 30


def _offsets(sizes):
    return torch.tensor([0] + sizes, device="cuda").cumsum(0).to(torch.int32)


def _scales(dtype, x, w):
    if dtype != "e4m3":
        return {}
    return dict(x_scale=torch.ones(x.shape[0], device="cuda"),
                w_scale=torch.ones(w.shape[:2], device="cuda"))


# rows of the last group, and of the first, so that the rule takes each kernel
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows,kind", [(150, "rows2"), (150, "rows4"), (2800, "ring"),
                                       (21000, "tiles")])
@pytest.mark.parametrize("up", [False, True])
def test_grouped_weights_past_4_gib_in_every_kernel(lk, dtype, rows, kind, up):  # noqa: F811
    """a matrix a group, the last ones behind 4 GiB: rows of every row tile, all columns"""
    d_in = 8192 if kind != "rows2" else 2048
    d_out = 2048
    G = 5 * GIB // (d_in * d_out * P.BYTES[dtype])
    sizes = [rows // 3] + [0] * (G - 2) + [rows - rows // 3]
    got = P.plan(dtype, up, sizes, d_in, d_out)
    _say("far weights", dtype, rows, up, G, P.kind(got))
    assert (P.kind(got) or "").split(" ")[0].startswith(kind)
    g = torch.Generator(device="cuda").manual_seed(31)
    x = _whole(g, (rows, d_in), TYPE[dtype])
    w = torch.zeros((G, d_out, d_in), dtype=TYPE[dtype], device="cuda")
    kw = _scales(dtype, x, w)
    ends = [_whole(g, (d_out, d_in), torch.float32) for _ in range(2)]
    w[0], w[G - 1] = ends[0].to(w.dtype), ends[1].to(w.dtype)
    if up:   # the gate is so large that silu leaves it as it is, or gives 0
        kw["w_up"] = torch.zeros_like(w)
        kw["w_up"][0, :, 0] = kw["w_up"][G - 1, :, 0] = 1
        if dtype == "e4m3":
            kw["w_up_scale"] = kw["w_scale"]
    out = torch.full((rows, d_out), -9.0, dtype=BF, device="cuda")
    lk.grouped_product(x, w, _offsets(sizes), out, **kw)
    at = torch.arange(0, rows, 1 if rows < 3000 else 13, device="cuda")
    first = at < rows // 3
    xs = x[at].double()
    want = torch.where(first[:, None], xs @ ends[0].double().T, xs @ ends[1].double().T)
    if up:
        want = want / (1 + torch.exp(-want)) * xs[:, :1]
        bound = (2.0 ** -20 + 2.0 ** -8 * 1.01) * want.abs() + 2.0 ** -99
        assert ((out[at].double() - want).abs() <= bound).all()
    else:
        assert torch.equal(out[at], want.to(BF))


@pytest.mark.parametrize("dtype", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("gib,kind", [(1.9, "tiles"), (3.9, "tiles"), (4.2, "ring")])
def test_grouped_gathers_from_rows_around_2_and_4_gib(lk, dtype, gib, kind):  # noqa: F811
    """the large tiles' offsets have 32 bits, the sign bit set from 2 GiB on; from 4 GiB on the
    rows go to another kernel"""
    row, d_out = 2048, 2048
    d_in = row // P.BYTES[dtype]
    x_rows = int(gib * GIB) // row
    sizes = [4000, 3000, 0, 5003, 3809]
    m = sum(sizes)
    got = P.plan(dtype, False, sizes, d_in, d_out, 1, x_rows)
    _say("far rows", dtype, gib, P.kind(got))
    assert P.kind(got).startswith(kind)
    g = torch.Generator(device="cuda").manual_seed(32)
    x = torch.empty((x_rows, d_in), dtype=TYPE[dtype], device="cuda")
    for a in range(0, x_rows, 1 << 18):
        x[a:a + (1 << 18)] = _whole(g, (min(1 << 18, x_rows - a), d_in), TYPE[dtype])
    w = _whole(g, (len(sizes), d_out, d_in), TYPE[dtype])
    rows = torch.randint(0, x_rows, (m,), generator=g, device="cuda", dtype=torch.int32)
    rows[::7] = x_rows - 1 - torch.arange(len(rows[::7]), device="cuda", dtype=torch.int32)
    off = _offsets(sizes)
    out = torch.empty((m, d_out), dtype=BF if dtype == "e4m3" else x.dtype, device="cuda")
    lk.grouped_product(x, w, off, out, rows=rows, picks=1, **_scales(dtype, x, w))
    for i in range(len(sizes)):
        a, b = int(off[i]), int(off[i + 1])
        want = x[rows[a:b].long()].double() @ w[i].double().T
        assert torch.equal(out[a:b], want.to(out.dtype)), f"group {i}"


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("groups,kind", [(3, "tiles"), (16384, "ring")])
def test_grouped_outputs_past_4_gib(lk, dtype, groups, kind):  # noqa: F811
    m, d_out, d_in = 16384 * 36, 4096, 128
    sizes = [m // groups] * groups
    assert P.kind(P.plan(dtype, False, sizes, d_in, d_out)).startswith(kind)
    _say("far outputs", dtype, groups)
    g = torch.Generator(device="cuda").manual_seed(33)
    x, w = _whole(g, (m, d_in), TYPE[dtype]), _whole(g, (1, d_out, d_in), TYPE[dtype])
    w = w.expand(groups, -1, -1).contiguous()
    out = torch.empty((m, d_out), dtype=BF, device="cuda")
    lk.grouped_product(x, w, _offsets(sizes), out, **_scales(dtype, x, w))
    for a in range(0, m, 1 << 16):
        at = torch.arange(a, min(m, a + (1 << 16)), 5, device="cuda")
        assert torch.equal(out[at], (x[at].double() @ w[0].double().T).to(BF)), f"rows from {a}"
