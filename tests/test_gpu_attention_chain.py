"""An attention sublayer as a decoder runs it: norm, a packed product of q, k and v,
head norms with positions, the cache, attention, the output projection, and the
injection set that the layer's Delta selects; captured graphs, streams, operands far
apart."""

import pytest
import torch

from paper_2607_16305_amd import lookme as lk
from tests import attention as A
from tests import operators as R

pytestmark = pytest.mark.gpu

I32, BF = torch.int32, torch.bfloat16
HQ, HK, D, W, PAGE = 8, 2, 64, 512, 32
SCALE = D ** -0.5


def _gen(seed=0):
    return torch.Generator().manual_seed(seed)


def _close(got, want):
    v, e = want
    far = (got.cpu().double() - v).abs() - e
    assert not far.isnan().any() and far.max() <= 0, f"{far.max()} past the bound"


def _quantized(g, d_out, d_in):
    q = torch.randint(0, 16, (d_out, d_in), generator=g)
    s = ((0.5 + torch.rand((d_out, d_in // 64), generator=g)) * 0.2 * d_in ** -0.5).to(BF)
    return R.pack(q), s


class Layer:
    """Weights, a cache and the buffers of up to n rows"""

    def __init__(self, n, pages, seed=0):
        g = _gen(seed)
        self.w = {"norm": (1 + 0.1 * torch.randn(W, generator=g)).to(BF),
                  "qkv": _quantized(g, (HQ + 2 * HK) * D, W), "o": _quantized(g, W, HQ * D),
                  "q": (1 + 0.1 * torch.randn(D, generator=g)).to(BF),
                  "k": (1 + 0.1 * torch.randn(D, generator=g)).to(BF),
                  "freq": torch.tensor([1e4 ** (-i / 32) for i in range(32)])}
        on = lambda x: tuple(t.cuda() for t in x) if isinstance(x, tuple) else x.cuda()  # noqa: E731
        self.g = {k: on(v) for k, v in self.w.items()}
        self.cache = torch.full(lk.cache_shape(pages, HK, PAGE, D), 255, dtype=torch.uint8,
                                device="cuda")
        e = lambda *s: torch.zeros(s, dtype=BF, device="cuda")  # noqa: E731
        self.y, self.packed = e(n, W), e(n, HQ + 2 * HK, D)
        self.q, self.att, self.delta = e(n, HQ, D), e(n, HQ, D), e(n, W)
        self.ws = torch.empty(lk.LOOKME_ATTENTION_WORKSPACE, dtype=torch.uint8, device="cuda")

    def run(self, hidden, pos, slots, lengths, pages, q_offsets=None, stream=None):
        """Delta of hidden [n, W]; nothing here waits for the GPU"""
        n, g, st = hidden.shape[0], self.g, dict(stream=stream)
        y, packed, q, att = self.y[:n], self.packed[:n], self.q[:n], self.att[:n]
        lk.residual_norm(hidden, weight=g["norm"], out=y, **st)
        lk.quant_product(y, *g["qkv"], packed.view(n, -1), **st)
        k, v = packed[:, HQ:HQ + HK], packed[:, HQ + HK:]
        lk.head_norm_rotary(packed[:, :HQ], q, k=k, k_out=k, q_weight=g["q"], k_weight=g["k"],
                            pos=pos, freq=g["freq"], **st)
        lk.cache_write(k, v, slots, self.cache, **st)
        lk.cache_attention(q, self.cache, pages, lengths, att, self.ws, q_offsets=q_offsets, **st)
        lk.quant_product(att.view(n, -1), *g["o"], self.delta[:n], **st)
        return self.delta[:n]


def _tables(lengths, width):
    """page tables of sequences that take turns in a cache"""
    B = len(lengths)
    t = torch.arange(width)[None] * B + torch.arange(B)[:, None]
    return t.to(I32)


def _slots(table, b, t):
    return table[b, t // PAGE] * PAGE + t % PAGE


def test_a_sublayer_through_prefill_and_decode():
    first = [70, 33, 5]
    table = _tables(first, 4)
    n = sum(first)
    layer = Layer(n, 12)
    seq = torch.cat([torch.full((m,), b) for b, m in enumerate(first)])
    at = torch.cat([torch.arange(m) for m in first])
    seen = [(torch.zeros((0, HK, D), dtype=torch.float64),) * 2 for _ in first]
    lengths = torch.tensor(first, dtype=I32)
    for turn in range(4):                  # a prefill and three decoded tokens
        if turn:
            seq, at = torch.arange(3), lengths.long()
            lengths = lengths + 1
        rows = len(seq)
        hidden = torch.randn((rows, W), generator=_gen(turn)).to(BF)
        counts = torch.bincount(seq, minlength=3)
        off = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)]).to(I32)
        slots = torch.stack([_slots(table, b, t) for b, t in zip(seq, at)]).to(I32)
        delta = layer.run(hidden.cuda(), at.to(I32).cuda(), slots.cuda(), lengths.cuda(),
                          table.cuda(), None if turn else off.cuda())
        w, host = layer.w, lambda t: t[:rows].cpu()  # noqa: E731
        y = host(layer.y)
        v, e = R.norm(hidden, w["norm"], 1e-6)
        _close(y, (v, e + 2.0 ** -8 * v.abs() * (1 + 2.0 ** -7)))
        # the packed rows: k was normed and turned in place, v is as the product gave it
        v, e = R.quant(y, *w["qkv"])
        v, e = v.view(rows, -1, D), e.view(rows, -1, D)
        packed = host(layer.packed)
        _close(packed[:, HQ + HK:], (v[:, HQ + HK:], e[:, HQ + HK:]))
        # what the cache holds of these rows is what came out of the norm
        k, val = packed[:, HQ:HQ + HK], packed[:, HQ + HK:]
        rk, rv = A.read(layer.cache.cpu(), slots)
        assert torch.equal(rk, A.value(*A.quantize(k))) and torch.equal(rv, A.value(*A.quantize(val)))
        q, att = host(layer.q), host(layer.att)
        for b in range(3):
            mine = seq == b
            seen[b] = (torch.cat([seen[b][0], rk[mine]]), torch.cat([seen[b][1], rv[mine]]))
            _close(att[mine], A.attention(q[mine], *seen[b], SCALE, True))
        _close(delta, R.quant(att.view(rows, -1), *w["o"]))
    # the same rows' head norms, from the product computed again
    again = torch.zeros_like(layer.packed[:3])
    lk.quant_product(layer.y[:3], *layer.g["qkv"], again.view(3, -1))
    again = again.cpu()
    for got, x, weight in ((layer.q[:3], again[:, :HQ], "q"),
                           (layer.packed[:3, HQ:HQ + HK], again[:, HQ:HQ + HK], "k")):
        _close(got, A.rotary(x, weight=layer.w[weight], eps=1e-6, pos=at.to(I32),
                             freq=layer.w["freq"]))


def test_delta_selects_the_injection_set():
    """the sublayer's output is the crit of lookme_select"""
    n, keep = 60, 15
    layer = Layer(n, 4)
    hidden = (torch.randn((n, W), generator=_gen(5)) *
              torch.logspace(-1, 1, n)[torch.randperm(n, generator=_gen(6)), None]).to(BF)
    table = torch.arange(4, dtype=I32)[None]
    at = torch.arange(n, dtype=I32)
    delta = layer.run(hidden.cuda(), at.cuda(), at.cuda(), torch.tensor([n], dtype=I32).cuda(),
                      table.cuda(), torch.tensor([0, n], dtype=I32).cuda())
    g = _gen(7)
    t = lk.Table(torch.randn((4, 64), generator=g).to(BF).cuda(),
                 torch.randn((4, 8, 64), generator=g).to(BF).cuda(),
                 torch.randn((32, 64), generator=g).to(BF).cuda(), 2)
    kept = torch.zeros(keep, dtype=I32, device="cuda")
    t.select(delta, kept, keep)
    norms = delta.cpu().double().square().sum(1)
    want = norms.topk(keep + 1).values
    assert want[keep - 1] > want[keep] * (1 + 1e-5)
    assert kept.cpu().tolist() == norms.topk(keep).indices.sort().values.tolist()


def _decode_inputs(B, lengths, width, seed):
    table = _tables(lengths, width)
    hidden = torch.randn((B, W), generator=_gen(seed)).to(BF)
    at = torch.tensor(lengths) - 1
    slots = torch.stack([_slots(table, b, t) for b, t in enumerate(at)])
    return [t.cuda() for t in (hidden, at.to(I32), slots.to(I32),
                               torch.tensor(lengths, dtype=I32), table)]


def test_captured_decode_steps():
    """Two graphs that share a workspace, replayed by turns with other inputs, eager work
    and synchronizations between them"""
    B, width = 3, 40
    layer, other = Layer(B, B * width), Layer(B, B * width, seed=3)
    other.ws = layer.ws
    filled = [900, 37, 1200]
    for l in (layer, other):               # tokens before the steps
        for b, m in enumerate(filled):
            t = torch.arange(m)
            table = _tables(filled, width)
            slots = (table[b, t // PAGE] * PAGE + t % PAGE).to(I32).cuda()
            k = torch.randn((m, HK, D), generator=_gen(b)).to(BF).cuda()
            lk.cache_write(k, k.flip(2).contiguous(), slots, l.cache)
    static = [_decode_inputs(B, [m + 1 for m in filled], width, 0) for _ in range(2)]
    for l, s in zip((layer, other), static):
        l.run(*s)
    torch.cuda.synchronize()
    graphs = []
    for l, s in zip((layer, other), static):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            l.run(*s)
        graphs.append(g)
    for step in range(5):
        for which, (l, s, g) in enumerate(zip((layer, other), static, graphs)):
            new = _decode_inputs(B, [m + 1 + step for m in filled], width, 10 * step + which)
            for a, b in zip(s, new):
                a.copy_(b)
            g.replay()
            got = (l.delta.clone(), l.cache.clone())
            l.delta.zero_()
            eager = l.run(*new)
            assert torch.equal(got[0], eager) and torch.equal(got[1], l.cache)
            assert got[0].isfinite().all() and got[0].any()
        torch.cuda.synchronize()


def test_calls_on_another_stream():
    B, width = 2, 8
    layer = Layer(B, B * width)
    args = _decode_inputs(B, [1, 1], width, 0)
    want = layer.run(*args).clone()
    layer.cache.fill_(255)
    layer.delta.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = layer.run(*args, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    layer.delta.zero_()
    layer.cache.fill_(255)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer.run(*args)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_two_calls_at_once_with_a_workspace_each():
    """the same rows on two streams, long enough to be cut into parts"""
    B, width = 4, 300
    layer = Layer(B, B * width)
    n = [9000, 1, 4000, 9600]
    k = torch.randn((B * width * PAGE, HK, D), generator=_gen(2)).to(BF).cuda()
    lk.cache_write(k, k, torch.arange(B * width * PAGE, dtype=I32).cuda(), layer.cache)
    q = torch.randn((B, HQ, D), generator=_gen(3)).to(BF).cuda()
    table, lengths = _tables(n, width).cuda(), torch.tensor(n, dtype=I32).cuda()
    need = lk.lookme_cache_attention_workspace(lk.LOOKME_BF16, B, B, HQ, HK, D, width, PAGE)
    assert 0 < need < lk.LOOKME_ATTENTION_WORKSPACE
    outs, streams = [torch.zeros_like(q) for _ in range(3)], [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    lk.cache_attention(q, layer.cache, table, lengths, outs[2], layer.ws)
    torch.cuda.synchronize()
    for _ in range(10):
        for o, w, s in zip(outs, ws, streams):
            lk.cache_attention(q, layer.cache, table, lengths, o, w, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[2])
    with pytest.raises(lk.LookmeError) as e:
        lk.cache_attention(q, layer.cache, table, lengths, outs[0], ws[0][:need - 256])
    assert e.value.status == lk.LOOKME_ERR_WORKSPACE


def test_a_cache_and_rows_past_4_gib():
    g = _gen(4)
    d, pages = 128, 1_050_000                        # 4.6 GB of pages of 32 tokens
    cache = torch.empty(lk.cache_shape(pages, 1, 32, d), dtype=torch.uint8, device="cuda")
    step = ((1 << 30) + 64) // 2 + 8 * 64            # rows 1 GiB and more apart in bytes
    wide = torch.empty(5 * step + 4096, dtype=BF, device="cuda")
    k = wide.as_strided((5, 1, d), (step, d, 1))
    v = wide[1024:].as_strided((5, 1, d), (step, d, 1))
    kv = torch.randn((2, 5, 1, d), generator=g).to(BF)
    k.copy_(kv[0])
    v.copy_(kv[1])
    tok = torch.tensor([pages * 32 - 1, pages * 32 - 2, 0, 1_000_000 * 32 + 7, 5], dtype=I32)
    lk.cache_write(k, v, tok.cuda(), cache)
    out = wide[2048:].as_strided((5, 1, d), (step, d, 1))
    out2 = torch.zeros((5, 1, d), dtype=BF, device="cuda")
    lk.cache_read(tok.cuda(), cache, out, out2)
    assert torch.equal(out.cpu().double(), A.value(*A.quantize(kv[0])))
    assert torch.equal(out2.cpu().double(), A.value(*A.quantize(kv[1])))
    # attention over a page behind 4 GiB, of rows far apart
    n = 32
    kk, vv = torch.randn((n, 1, d), generator=g), torch.randn((n, 1, d), generator=g)
    slots = (pages - 3) * 32 + torch.arange(n)
    lk.cache_write(kk.cuda(), vv.cuda(), slots.to(I32).cuda(), cache)
    q = wide[2560:].as_strided((5, 1, d), (step, d, 1))
    qc = torch.randn((5, 1, d), generator=g).to(BF)
    q.copy_(qc)
    ws = torch.empty(lk.LOOKME_ATTENTION_WORKSPACE, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[pages - 3]], dtype=I32).cuda()
    lk.cache_attention(q, cache, table, torch.tensor([n], dtype=I32).cuda(), q, ws,
                       q_offsets=torch.tensor([0, 5], dtype=I32).cuda())
    _close(q, A.attention(qc, A.value(*A.quantize(kk)), A.value(*A.quantize(vv)), d ** -0.5, True))
    x = q.clone()
    pos, freq = torch.arange(5, dtype=I32), torch.rand(64, generator=g)
    lk.head_norm_rotary(q, q, pos=pos.cuda(), freq=freq.cuda())
    _close(q, A.rotary(x.cpu(), eps=1e-6, pos=pos, freq=freq))


def test_more_rows_than_a_launch_and_many_sequences():
    n = (1 << 22) + 5
    x = torch.randn((64, 1, 8), generator=_gen(1)).repeat(n // 64 + 1, 1, 1)[:n].to(BF)
    pos = torch.arange(n, dtype=I32)
    freq = torch.tensor([1.0, 0.1, 0.01, 0.001])
    out = torch.empty((n, 1, 8), dtype=BF, device="cuda")
    lk.head_norm_rotary(x.cuda(), out, pos=pos.cuda(), freq=freq.cuda())
    for a, b in ((0, 100), ((1 << 22) - 50, n)):
        _close(out[a:b], A.rotary(x[a:b], eps=1e-6, pos=pos[a:b], freq=freq))
    # 3000 sequences of one token or none, and some that are longer
    B, g = 3000, _gen(2)
    lengths = torch.randint(0, 3, (B,), generator=g)
    lengths[::500] = 90
    table = torch.randint(0, 16, (B, 3), generator=g, dtype=I32)
    k, v = torch.randn((512, 1, 64), generator=g), torch.randn((512, 1, 64), generator=g)
    cache = torch.zeros(lk.cache_shape(16, 1, 32, 64), dtype=torch.uint8, device="cuda")
    lk.cache_write(k.cuda(), v.cuda(), torch.arange(512, dtype=I32).cuda(), cache)
    kd, vd = A.value(*A.quantize(k)), A.value(*A.quantize(v))
    q = torch.randn((B, 2, 64), generator=g).to(BF)
    out = torch.full_like(q, 7).cuda()
    ws = torch.empty(lk.LOOKME_ATTENTION_WORKSPACE, dtype=torch.uint8, device="cuda")
    lk.cache_attention(q.cuda(), cache, table.cuda(), lengths.to(I32).cuda(), out, ws)
    for b in list(range(0, B, 500)) + list(range(1, 60)):
        t = torch.arange(int(lengths[b]))
        at = table[b, t // 32].long() * 32 + t % 32
        _close(out[b:b + 1], A.attention(q[b:b + 1], kd[at], vd[at], 0.125, True))
    assert not out[(lengths == 0).cuda()].any()
