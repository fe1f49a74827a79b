"""The operators around a LookME layer as they are used together: routed tokens
through their experts and back into the hidden states, decoded tokens through
4-bit weights, captured into graphs, on other streams and beside each other."""

import pytest
import torch

from tests import operators as R

pytestmark = pytest.mark.gpu

BF, F32, E4M3, I32 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.int32
EPS = 1e-6


@pytest.fixture(scope="module")
def lk():
    from paper_2607_16305_amd import lookme
    assert torch.cuda.is_available(), "no GPU visible"
    lookme.load()
    return lookme


def _say(*a):
    print("[gpu-operators]", *a, flush=True)


def _rand(seed, *shape, std=1.0, dtype=BF):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype)


def _close(got, want, bound, what):
    bad = ~((got.double().cpu() - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} values"


class Experts:
    """n tokens, k picks each of E experts (SwiGLU, then down), weighted back into
    the hidden states, normed and quantised for a product per scene: every
    buffer that the calls use."""

    def __init__(self, n=300, k=2, E=8, d=256, d_ff=192, seed=0):
        r = lambda i, *s, **kw: _rand(seed + i, *s, **kw).cuda()  # noqa: E731
        self.n, self.k, self.E = n, k, E
        self.x, self.hidden = r(1, n, d), r(2, n, d)
        self.gate, self.up = r(3, E, d_ff, d, std=d ** -0.5), r(4, E, d_ff, d, std=d ** -0.5)
        self.down = r(5, E, d, d_ff, std=d_ff ** -0.5)
        self.norm_w = r(6, d)
        # the router: one scene whose primitives are the experts
        self.keys = r(7, 1, E, d, std=d ** -0.5)
        self.next_w, self.next_s = (t.cuda() for t in R.quantize_rows(
            _rand(seed + 8, E, 128, d, std=d ** -0.5)))
        e = lambda *s, dtype=BF: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
        self.q, self.scene = e(n, d), e(n, dtype=I32)
        self.prim, self.w = e(n, k, dtype=I32), e(n, k, dtype=F32)
        self.rows, self.offsets = e(n * k, dtype=I32), e(E + 1, dtype=I32)
        self.u, self.y = e(n * k, d_ff), e(n * k, d)
        self.hidden_out, self.quant, self.scale = e(n, d), e(n, d, dtype=E4M3), e(n, dtype=F32)
        self.last = e(n * k, 128)

    def route(self, lk):
        """the framework's own lookup picks the experts and their weights"""
        self.table = lk.Table(self.keys[:, 0].contiguous(), self.keys, self.keys[0], self.k)
        self.scene.zero_()
        self.table.reserve(1, self.n)
        self.table.lookup(self.x, self.scene, self.prim, self.w)

    def run(self, lk, stream=None):
        n, k = self.n, self.k
        lk.group_rows(self.prim, self.E, self.rows, self.offsets, stream=stream)
        lk.grouped_product(self.x, self.gate, self.offsets, self.u, rows=self.rows, picks=k,
                           w_up=self.up, stream=stream)
        lk.grouped_product(self.u, self.down, self.offsets, self.y, rows=self.rows, picks=0,
                           scatter=True, stream=stream)
        lk.residual_norm(self.hidden, weight=self.norm_w, eps=EPS, add=self.y.view(n, k, -1),
                         part_w=self.w, hidden_out=self.hidden_out, out_quant=self.quant,
                         scale_out=self.scale, stream=stream)
        lk.grouped_product(self.quant, self.next_w, self.offsets, self.last, rows=self.rows,
                           picks=k, scatter=True, x_scale=self.scale, w_scale=self.next_s,
                           stream=stream)

    def outputs(self):
        return [t.clone() for t in (self.offsets, self.y, self.hidden_out, self.quant.view(torch.uint8),
                                    self.scale, self.last)]

    def check(self):
        c = lambda t: t.cpu()  # noqa: E731
        rows, off, n, k = c(self.rows), c(self.offsets), self.n, self.k
        want, offsets = R.group_rows(c(self.prim).flatten(), self.E)
        assert off.tolist() == offsets and rows[:len(want)].tolist() == want
        m, kept = n * k, rows[:len(want)].long()
        u, e = R.grouped(c(self.x), c(self.gate), off, m, rows, k, c(self.up))
        _close(self.u[:len(want)], u[:len(want)], e[:len(want)], "gate and up")
        y, e = R.grouped(c(self.u), c(self.down), off, m, rows, 0, None, True)
        _close(self.y[kept.cuda()], y[kept], e[kept], "down")
        s, e = R.residual_sum(c(self.hidden), c(self.y).view(n, k, -1), c(self.w))
        _close(self.hidden_out, s, e, "residual")
        v, e = R.norm(c(self.hidden_out), c(self.norm_w), EPS)
        sc = c(self.scale).double()
        _close(self.scale, v.abs().amax(1) / 448, 64 * R.U32 * v.abs().amax(1) / 448, "scale")
        v = v / sc[:, None]
        _close(self.quant.float(), v, (2.0 ** -4 + 2.0 ** -16) * v.abs() + 2.0 ** -10, "quant")
        z, e = R.grouped(c(self.quant), c(self.next_w), off, m, rows, k, None, True,
                         c(self.scale), c(self.next_s), None, BF)
        _close(self.last[kept.cuda()], z[kept], e[kept], "the next product")


@pytest.mark.parametrize("n,k,E", [(1, 2, 8), (5, 1, 3), (300, 2, 8), (700, 4, 16)])
def test_routed_tokens_through_their_experts(lk, n, k, E):
    _say("experts", n, k, E)
    s = Experts(n, k, E)
    s.route(lk)
    s.run(lk)
    torch.cuda.synchronize()
    s.check()


def test_route_of_scenes_groups_their_rows(lk):
    """lookme_route's scenes, with the balancing bias, as the groups of a product"""
    n, S, d = 400, 12, 64
    x, keys = _rand(1, n, d).cuda(), _rand(2, S, d).cuda()
    table = lk.Table(keys, keys[:, None].contiguous(), keys, 1)
    q, scene = torch.empty_like(x), torch.empty((n,), dtype=I32, device="cuda")
    table.route(x, None, q, scene)
    rows = torch.empty((n,), dtype=I32, device="cuda")
    off = torch.empty((S + 1,), dtype=I32, device="cuda")
    lk.group_rows(scene, S, rows, off)
    w, out = _rand(3, S, 32, d).cuda(), torch.empty((n, 32), dtype=BF, device="cuda")
    lk.grouped_product(x, w, off, out, rows=rows, scatter=True)
    xs, ws = x.cpu().double(), w.cpu().double()[scene.cpu().long()]
    want = (ws @ xs[:, :, None])[:, :, 0]
    bound = (d + 4) * R.U32 * (ws.abs() @ xs.abs()[:, :, None])[:, :, 0]
    _close(out, want, bound + R.HALF[BF] * 1.01 * want.abs(), "out")


def test_masked_tokens_keep_their_hidden_states(lk):
    """a token without experts (ids -1, weights 0): its entries' rows are never
    written, hold NaN here, and leave its hidden state's bits alone"""
    s = Experts()
    s.route(lk)
    s.prim[7] = -1
    s.prim[123, 1] = -1
    s.w[7] = 0
    s.w[123, 1] = 0
    s.prim[299], s.w[299] = s.E, 0
    for t in (s.u, s.y, s.last):
        t.fill_(float("nan"))
    s.run(lk)
    torch.cuda.synchronize()
    for row in (7, 299):
        assert torch.equal(s.hidden_out[row], s.hidden[row])
        assert s.y.view(s.n, s.k, -1)[row].isnan().all()
        assert s.last.view(s.n, s.k, -1)[row].isnan().all()
    assert not s.hidden_out.isnan().any()
    s.check()


class Decode:
    """n decoded tokens through norm, gate and up, and down on 4-bit weights."""

    def __init__(self, n, d=512, d_ff=320, group=64, dtype=BF, seed=50):
        g = torch.Generator().manual_seed(seed)
        self.hidden, self.norm_w = _rand(seed, n, d, dtype=dtype), _rand(seed + 1, d, dtype=dtype)
        mat = lambda o, i: (  # noqa: E731
            torch.randint(0, 256, (o, i // 2), generator=g, dtype=torch.uint8),
            ((torch.rand((o, i // group), generator=g) + 0.5) * 0.2 * i ** -0.5).to(dtype),
            torch.randint(0, 16, (o, i // group), generator=g, dtype=torch.uint8))
        self.mats = mat(d_ff, d), mat(d_ff, d), mat(d, d_ff)
        self.dev = [[t.cuda() for t in m] for m in self.mats]
        self.h, self.nw = self.hidden.cuda(), self.norm_w.cuda()
        self.x, self.u = torch.empty_like(self.h), torch.empty((n, d_ff), dtype=dtype, device="cuda")
        self.out = torch.empty_like(self.h)

    def run(self, lk, stream=None):
        a, b, c = self.dev
        lk.residual_norm(self.h, weight=self.nw, eps=EPS, out=self.x, stream=stream)
        lk.quant_swiglu(self.x, a[0], a[1], b[0], b[1], self.u, z_gate=a[2], z_up=b[2],
                        stream=stream)
        lk.quant_product(self.u, c[0], c[1], self.out, zero=c[2], add=self.h, stream=stream)

    def check(self):
        h = self.h.cpu()
        v, e = R.norm(h, self.norm_w, EPS)
        _close(self.x, v, e + R.HALF[h.dtype] * 1.01 * v.abs(), "norm")
        _close(self.u, *R.quant(self.x.cpu(), *self.mats[0], up=self.mats[1]), "gate and up")
        _close(self.out, *R.quant(self.u.cpu(), *self.mats[2], add=h), "down")


@pytest.mark.parametrize("n,dtype", [(1, BF), (3, F32), (40, BF)])
def test_decoded_tokens_on_small_weights(lk, n, dtype):
    _say("decode", n, dtype)
    s = Decode(n, dtype=dtype)
    s.run(lk)
    torch.cuda.synchronize()
    s.check()


def test_captured_and_replayed(lk):
    """two graphs, replayed in turn on new inputs, with eager calls between"""
    _say("graphs")
    a, b, eager = Experts(seed=0), Decode(2), Experts(n=40, k=1, seed=9)
    a.route(lk)
    eager.route(lk)
    graphs = []
    for s in (a, b):
        s.run(lk)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run(lk)
        graphs.append(g)
    for turn in range(3):
        a.x.copy_(_rand(100 + turn, *a.x.shape))
        a.prim.copy_(torch.randint(0, a.E, a.prim.shape, dtype=I32,
                                   generator=torch.Generator().manual_seed(turn)))
        b.h.copy_(_rand(200 + turn, *b.h.shape))
        for t in (a.y, a.hidden_out, a.last, b.out):
            t.zero_()
        torch.cuda.synchronize()
        graphs[0].replay()
        eager.run(lk)
        graphs[1].replay()
        torch.cuda.synchronize()
        a.check()
        b.check()
        eager.check()
        got = a.outputs()
        a.run(lk)
        torch.cuda.synchronize()
        for x, y in zip(got, a.outputs()):
            assert torch.equal(x, y), f"turn {turn}: replay and eager call differ"


def test_streams_beside_each_other(lk):
    """the same calls on two streams at once, on buffers of their own, give the
    bits they give alone; a stream given by argument or as the current one"""
    _say("streams")
    one, two = Experts(seed=0), Experts(n=500, k=4, seed=20)
    for s in (one, two):
        s.route(lk)
        s.run(lk)
    torch.cuda.synchronize()
    want = one.outputs(), two.outputs()
    for t in (one.y, one.last, two.y, two.last):
        t.zero_()
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        one.run(lk, stream=a)
        with torch.cuda.stream(b):
            two.run(lk)
    torch.cuda.synchronize()
    for s, w in zip((one, two), want):
        for x, y in zip(s.outputs(), w):
            assert torch.equal(x, y)


def test_entry_points_by_their_c_names(lk):
    """the raw bindings, with addresses and sizes"""
    h, out = _rand(1, 3, 64).cuda(), torch.empty((3, 64), dtype=BF, device="cuda")
    lk.lookme_residual_norm(lk.LOOKME_BF16, 3, 64, h, 0, None, None, None, EPS, None, out, None,
                            None)
    v, e = R.norm(h.cpu(), None, EPS)
    _close(out, v, e + R.HALF[BF] * 1.01 * v.abs(), "norm")
    pick = torch.tensor([1, 0, 1], dtype=I32, device="cuda")
    rows, off = torch.empty_like(pick), torch.empty((3,), dtype=I32, device="cuda")
    lk.lookme_group_rows(2, 3, pick, rows, off)
    assert rows.tolist() == [1, 0, 2] and off.tolist() == [0, 1, 3]
    w = _rand(2, 2, 8, 64).cuda()
    y = torch.empty((3, 8), dtype=BF, device="cuda")
    lk.lookme_grouped_product(lk.LOOKME_BF16, 2, 3, 64, 8, h, 3, rows, 1, off, w, None, y, 1)
    _close(y, *R.grouped(h.cpu(), w.cpu(), off.cpu(), 3, rows.cpu(), 1, None, True), "grouped")
    (hq, hs), (wq, ws) = R.quantize_rows(h.cpu()), R.quantize_rows(w.cpu())
    dev = [t.cuda() for t in (hq, hs, wq, ws)]
    lk.lookme_grouped_product_quant(2, 3, 64, 8, dev[0], dev[1], 3, rows, 1, off, dev[2], dev[3],
                                    None, None, y, 1)
    _close(y, *R.grouped(hq, wq, off.cpu(), 3, rows.cpu(), 1, None, True, hs, ws, None, BF),
           "grouped e4m3")
    s = Decode(3, d=64, d_ff=32, group=32)
    a, b, c = s.dev
    u, z = torch.empty((3, 32), dtype=BF, device="cuda"), torch.empty((3, 64), dtype=BF, device="cuda")
    lk.lookme_quant_swiglu(lk.LOOKME_BF16, 3, 64, 32, 32, h, a[0], a[1], a[2], b[0], b[1], b[2], u)
    _close(u, *R.quant(h.cpu(), *s.mats[0], up=s.mats[1]), "swiglu")
    lk.lookme_quant_product(lk.LOOKME_BF16, 3, 32, 64, 32, u, c[0], c[1], c[2], h, z)
    _close(z, *R.quant(u.cpu(), *s.mats[2], add=h.cpu()), "product")
