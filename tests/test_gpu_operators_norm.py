"""GPU tests of the residual norm of a sum that is not stored."""

import pytest
import torch

from tests.test_gpu_operators import BF, DT, E4M3, _check_norm, _rand, _say, lk  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [512, 1160, 4096, 8184, 16384, 40000])
@pytest.mark.parametrize("parts,weighted", [(1, False), (1, True), (2, True), (5, False)])
@pytest.mark.parametrize("n", [3, 300])
def test_norm_of_a_sum_that_is_not_stored(lk, dtype, d, parts, weighted, n):  # noqa: F811
    """the same bits in out, out_quant and scale_out as beside a stored sum (which is
    compared with the plain form), all outputs together and one by one"""
    _say("norm without its sum", dtype, n, d, parts, weighted)
    dt = DT[dtype]
    h, add = _rand(1, n, d, std=2.0, dtype=dt), _rand(2, n, parts, d, dtype=dt)
    pw = torch.softmax(_rand(3, n, parts), 1) * 1.5 if weighted else None
    if weighted:
        pw[1, 0] = 0
        add[1, 0] = float("nan")
    g = _rand(4, d, dtype=dt)
    hd, ad, gd, pd = h.cuda(), add.cuda(), g.cuda(), None if pw is None else pw.cuda()

    def run(store, out, quant):
        o = torch.full_like(hd, 7.0) if out else None
        q = torch.zeros((n, d), dtype=E4M3, device="cuda") if quant else None
        sc = torch.zeros((n,), device="cuda") if quant else None
        ho = torch.empty_like(hd) if store else None
        lk.residual_norm(hd, weight=gd, eps=1e-6, add=ad, part_w=pd, hidden_out=ho, out=o,
                         out_quant=q, scale_out=sc)
        return ho, o, q, sc

    ho, o, q, sc = run(True, True, True)
    _check_norm(h, add, pw, g, ho, o, q, sc)
    for out, quant in ((True, True), (True, False), (False, True)):
        _, o1, q1, sc1 = run(False, out, quant)
        if out:
            assert torch.equal(o1.view(torch.uint8), o.view(torch.uint8))
        if quant:
            assert torch.equal(q1.view(torch.uint8), q.view(torch.uint8))
            assert torch.equal(sc1, sc)
    assert torch.equal(hd.cpu(), h) and torch.equal(ad.cpu().nan_to_num(), add.nan_to_num())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [512, 4096, 40000])
def test_norm_of_rows_whose_squares_leave_float32(lk, dtype, d):  # noqa: F811
    """values from 2^64 on give 0, of 2^63 the norm; a row beside them is its own"""
    _say("norm of huge rows", dtype, d)
    h = torch.ones((4, d), dtype=DT[dtype])
    h[1], h[2, 1:] = 2.0 ** 64, 0
    h[2, 0] = 2.0 ** 63
    hd = h.cuda()
    o = torch.full_like(hd, 7.0)
    q, sc = torch.zeros((4, d), dtype=E4M3, device="cuda"), torch.zeros(4, device="cuda")
    lk.residual_norm(hd, eps=0.0, out=o, out_quant=q, scale_out=sc)
    assert (o[1] == 0).all() and (q[1].float() == 0).all() and float(sc[1]) == 2.0 ** -126
    assert torch.equal(o[0], o[3]) and ((o[0].double() - 1).abs() <= 2.0 ** -8).all()
    assert abs(float(o[2, 0]) / d ** 0.5 - 1) <= 2.0 ** -8 and (o[2, 1:] == 0).all()
