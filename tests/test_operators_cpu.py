"""The operators around a LookME layer without a GPU: argument checks of their
entry points before anything is launched (stand-in device addresses, never
dereferenced), and the checks of the torch bindings."""

import pytest
import torch

from paper_2607_16305_amd import lookme as lk
from tests import operators as R

A = 0x7F0000100000     # an aligned stand-in address
OK, INVALID, UNSUPPORTED = lk.LOOKME_OK, lk.LOOKME_ERR_INVALID, lk.LOOKME_ERR_UNSUPPORTED
BF, F32 = lk.LOOKME_BF16, lk.LOOKME_F32
E4M3 = torch.float8_e4m3fn


def _status(fn, *a, **kw):
    try:
        fn(*a, **kw)
    except lk.LookmeError as e:
        assert str(e)
        return e.status
    return OK


def _norm(dtype=BF, n=4, d=64, hidden=A, parts=1, add=A, part_w=None, weight=A, eps=1e-6,
          hidden_out=A, out=None, out_quant=None, scale_out=None):
    return _status(lk.lookme_residual_norm, dtype, n, d, hidden, parts, add, part_w, weight, eps,
                   hidden_out, out, out_quant, scale_out, 0)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), INVALID), (dict(n=-1), INVALID), (dict(n=2 ** 30 + 1), UNSUPPORTED),
    (dict(d=0), INVALID), (dict(d=60), UNSUPPORTED), (dict(dtype=F32, d=6), UNSUPPORTED),
    (dict(d=2 ** 24), UNSUPPORTED), (dict(parts=-1), INVALID), (dict(parts=0), INVALID),
    (dict(parts=0, add=None, part_w=A), INVALID), (dict(add=None), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(hidden=None), INVALID),
    (dict(hidden=A + 8), INVALID), (dict(weight=A + 2), INVALID), (dict(part_w=A + 4), INVALID),
    (dict(hidden_out=None), INVALID), (dict(out_quant=A), INVALID), (dict(scale_out=A), INVALID),
    (dict(out_quant=A, scale_out=A + 4), INVALID), (dict(out=A + 8), INVALID),
    (dict(n=0, hidden=None, add=None, hidden_out=None), OK)])
def test_residual_norm_refuses(kw, status):
    assert _norm(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(groups=0), INVALID), (dict(groups=lk.LOOKME_MAX_GROUPS + 1), UNSUPPORTED),
    (dict(n=-1), INVALID), (dict(n=2 ** 30 + 1), UNSUPPORTED), (dict(pick=None), INVALID),
    (dict(rows=A + 4), INVALID), (dict(offsets=None), INVALID),
    (dict(n=0, pick=None, rows=None, offsets=None), INVALID)])
def test_group_rows_refuses(kw, status):
    a = dict(groups=8, n=16, pick=A, rows=A, offsets=A)
    a.update(kw)
    assert _status(lk.lookme_group_rows, a["groups"], a["n"], a["pick"], a["rows"], a["offsets"],
                   0) == status


_GROUPED = [
    (dict(groups=0), INVALID), (dict(groups=lk.LOOKME_MAX_GROUPS + 1), UNSUPPORTED),
    (dict(m=-1), INVALID), (dict(m=2 ** 30 + 1), UNSUPPORTED), (dict(d_in=0), INVALID),
    (dict(d_in=20), UNSUPPORTED), (dict(d_out=0), INVALID), (dict(d_out=4), UNSUPPORTED),
    (dict(m=2 ** 30, d_out=2 ** 16), UNSUPPORTED),
    (dict(picks=-1), INVALID), (dict(picks=1, rows=None), INVALID),
    (dict(scatter=1, rows=None), INVALID), (dict(x_rows=15), INVALID), (dict(x_rows=-1), INVALID),
    (dict(x_rows=0, picks=2), INVALID), (dict(x_rows=2 ** 31), INVALID), (dict(x=None), INVALID),
    (dict(rows=A + 4), INVALID), (dict(offsets=None), INVALID), (dict(w=A + 8), INVALID),
    (dict(out=None), INVALID), (dict(m=0, x=None, w=None, out=None, offsets=None), OK)]


@pytest.mark.parametrize("kw,status", _GROUPED)
def test_grouped_product_refuses(kw, status):
    a = dict(dtype=BF, groups=8, m=16, d_in=64, d_out=32, x=A, x_rows=16, rows=A, picks=0,
             offsets=A, w=A, w_up=None, out=A, scatter=0)
    a.update(kw)
    assert _status(lk.lookme_grouped_product, *a.values(), 0) == status
    a.pop("dtype")
    q = {}
    for k, v in a.items():
        q[k] = v
        if k in ("x", "w"):
            q[k + "_scale"] = A
        if k == "w_up":
            q["up_scale"] = None
    assert _status(lk.lookme_grouped_product_quant, *q.values(), 0) == status
    if status == OK:
        return
    for bad in (dict(x_scale=None), dict(w_scale=A + 4), dict(up_scale=A), dict(w_up=A)):
        good = dict(zip(q, (8, 16, 64, 32, A, A, 16, A, 0, A, A, A, None, None, A, 0)))
        good.update(bad)
        assert _status(lk.lookme_grouped_product_quant, *good.values(), 0) == INVALID


def test_grouped_product_checks_its_dtype():
    assert _status(lk.lookme_grouped_product, 2, 8, 16, 64, 32, A, 16, None, 0, A, A, None, A, 0,
                   0) == INVALID


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), INVALID), (dict(n=-1), INVALID), (dict(n=2 ** 20), UNSUPPORTED),
    (dict(d_in=0), INVALID), (dict(group=0), INVALID), (dict(group=16), UNSUPPORTED),
    (dict(group=96), UNSUPPORTED), (dict(d_in=192, group=128), INVALID), (dict(d_out=0), INVALID),
    (dict(d_out=12), UNSUPPORTED), (dict(x=None), INVALID), (dict(w=A + 4), INVALID),
    (dict(scale=None), INVALID), (dict(zero=A + 1), INVALID), (dict(out=None), INVALID),
    (dict(n=0, x=None, w=None, scale=None, out=None), OK)])
def test_quant_products_refuse(kw, status):
    a = dict(dtype=BF, n=3, d_in=256, d_out=32, group=64, x=A, w=A, scale=A, zero=None, add=None,
             out=A)
    a.update(kw)
    assert _status(lk.lookme_quant_product, *a.values(), 0) == status
    both = [a[k] for k in ("dtype", "n", "d_in", "d_out", "group", "x", "w", "scale", "zero", "w",
                           "scale", "zero", "out")]
    assert _status(lk.lookme_quant_swiglu, *both, 0) == status
    if status == INVALID:
        good = [BF, 3, 256, 32, 64, A, A, A, None, A, A, None, A]
        for i in (9, 10):
            assert _status(lk.lookme_quant_swiglu, *good[:i], None, *good[i + 1:], 0) == INVALID


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


I32 = torch.int32


@pytest.mark.parametrize("call", [
    lambda: lk.residual_norm(_t(4, 64), out=_t(4, 64)),                        # on the CPU
    lambda: lk.residual_norm(_t(64), out=_t(64)),
    lambda: lk.residual_norm(_t(4, 64, dtype=torch.float16), out=_t(4, 64)),
    lambda: lk.residual_norm(_t(4, 128)[:, ::2], out=_t(4, 64)),               # strided
    lambda: lk.residual_norm(_t(4, 64), add=_t(4, 2, 32), out=_t(4, 64)),
    lambda: lk.residual_norm(_t(4, 64), add=_t(4, 64), part_w=_t(4, 2, dtype=torch.float32),
                             out=_t(4, 64)),
    lambda: lk.residual_norm(_t(4, 64), weight=_t(32), out=_t(4, 64)),
    lambda: lk.residual_norm(_t(4, 64), out_quant=_t(4, 64), scale_out=_t(4, dtype=torch.float32)),
    lambda: lk.group_rows(_t(8, dtype=torch.int64), 4, _t(8, dtype=I32), _t(5, dtype=I32)),
    lambda: lk.group_rows(_t(8, dtype=I32), 4, _t(7, dtype=I32), _t(5, dtype=I32)),
    lambda: lk.group_rows(_t(8, dtype=I32), 4, _t(8, dtype=I32), _t(4, dtype=I32)),
    lambda: lk.grouped_product(_t(8, 64), _t(2, 32, 32), _t(3, dtype=I32), _t(8, 32)),
    lambda: lk.grouped_product(_t(8, 64), _t(2, 32, 64), _t(2, dtype=I32), _t(8, 32)),
    lambda: lk.grouped_product(_t(8, 64), _t(2, 32, 64), _t(3, dtype=I32), _t(8, 16)),
    lambda: lk.grouped_product(_t(8, 64), _t(2, 32, 64), _t(3, dtype=I32), _t(8, 32),
                               rows=_t(9, dtype=I32)),
    lambda: lk.grouped_product(_t(8, 64), _t(2, 32, 64), _t(3, dtype=I32), _t(8, 32),
                               w_up=_t(2, 32, 32)),
    lambda: lk.grouped_product(_t(8, 64), _t(2, 32, 64), _t(3, dtype=I32), _t(8, 32),
                               x_scale=_t(8, dtype=torch.float32)),
    lambda: lk.grouped_product(_t(8, 64, dtype=E4M3), _t(2, 32, 64, dtype=E4M3),
                               _t(3, dtype=I32), _t(8, 32)),
    lambda: lk.grouped_product(_t(8, 64, dtype=E4M3), _t(2, 32, 64, dtype=E4M3),
                               _t(3, dtype=I32), _t(8, 32), x_scale=_t(8, dtype=torch.float32),
                               w_scale=_t(2, 16, dtype=torch.float32)),
    lambda: lk.quant_product(_t(2, 64), _t(8, 16, dtype=torch.uint8), _t(8, 2), _t(2, 8)),
    lambda: lk.quant_product(_t(2, 64), _t(8, 32, dtype=torch.uint8), _t(8, 3), _t(2, 8)),
    lambda: lk.quant_product(_t(2, 64), _t(8, 32, dtype=torch.uint8), _t(8, 2), _t(2, 16)),
    lambda: lk.quant_product(_t(2, 64), _t(8, 32, dtype=torch.uint8), _t(8, 2), _t(2, 8),
                             zero=_t(8, 1, dtype=torch.uint8)),
    lambda: lk.quant_product(_t(2, 64), _t(8, 32, dtype=torch.uint8),
                             _t(8, 2, dtype=torch.float32), _t(2, 8)),
    lambda: lk.quant_swiglu(_t(2, 64), _t(8, 32, dtype=torch.uint8), _t(8, 2),
                            _t(8, 32, dtype=torch.uint8), _t(8, 1), _t(2, 8)),
])
def test_bindings_refuse(call):
    assert _status(call) == INVALID


def test_plain_forms_agree_with_torch():
    """the float64 forms that the GPU tests compare with"""
    g = torch.Generator().manual_seed(0)
    q = torch.randint(0, 16, (8, 64), generator=g)
    assert torch.equal(R.unpack(R.pack(q)).long(), q)
    x = torch.randn((5, 64), generator=g)
    s = torch.rand((8, 2), generator=g)
    v, e = R.quant(x, R.pack(q), s)
    w = (q - 8).float() * s.repeat_interleave(32, 1)
    assert ((x @ w.T - v).abs() <= e).all()
    h, a = torch.randn((5, 64), generator=g), torch.randn((5, 3, 64), generator=g)
    y, e = R.residual_sum(h, a)
    assert ((h + a.sum(1) - y).abs() <= e).all()
    n, e = R.norm(h, None, 0.0)
    assert ((torch.nn.functional.rms_norm(h, (64,), eps=0.0) - n).abs() <= e).all()
    pick = torch.randint(-1, 6, (50,), generator=g, dtype=torch.int32)
    rows, off = R.group_rows(pick, 5)
    kept = ((pick >= 0) & (pick < 5)).nonzero()[:, 0]
    assert rows == kept[torch.sort(pick[kept], stable=True).indices].tolist()
    wm = torch.randn((5, 16, 64), generator=g)
    out, e = R.grouped(h.repeat(4, 1), wm, torch.tensor([0, 3, 3, 10, 11, 20]), 20)
    want = torch.cat([h.repeat(4, 1)[a:b] @ wm[i].T
                      for i, (a, b) in enumerate([(0, 3), (3, 3), (3, 10), (10, 11), (11, 20)])])
    assert ((want - out).abs() <= e).all()
    assert torch.equal(torch.tensor([r for r in rows]).sort().values, kept)
