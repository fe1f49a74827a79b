"""Attention's kernel of many rows on the GPU against a plain float64 form: whole keys
and cut ones, few sequences and more than a wave has lanes, blocks that are not finite,
pages out of range, captured graphs.  Every call asks the rule whether that kernel runs."""

import pytest
import torch

from paper_2607_16305_amd import lookme as lk
from tests import attention as A
from tests import attention_many as M

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
I32 = torch.int32
NAN = float("nan")


def _gen(seed=0):
    return torch.Generator().manual_seed(seed)


def _close(got, want):
    v, e = want
    far = (got.cpu().double() - v).abs() - e
    assert not far.isnan().any() and (far.numel() == 0 or far.max() <= 0), \
        f"{far.max()} past the bound"


class Call:
    """A call's inputs on the GPU.  Page 0 is no sequence's; it and what lies behind the
    lengths hold `garbage` (a byte, or None: any bytes)."""

    def __init__(self, name, dtype, d, seed=0, garbage=255, keys=1.5):
        self.seqs, self.hq, self.hkv, width, _ = M.CALLS[name]
        self.d, self.dt = d, DT[dtype]
        g = _gen(seed)
        used = [-(-n // M.PAGE) for _, n in self.seqs]
        self.num_pages = sum(used) + 1
        order = torch.randperm(self.num_pages - 1, generator=g) + 1
        shape = lk.cache_shape(self.num_pages, self.hkv, M.PAGE, d)
        cache = (torch.randint(0, 256, shape, generator=g, dtype=torch.uint8) if garbage is None
                 else torch.full(shape, garbage, dtype=torch.uint8))
        self.table = torch.full((len(self.seqs), width), -7, dtype=I32)
        self.slots, first = [], 0
        for b, (_, n) in enumerate(self.seqs):
            mine = order[first:first + used[b]]
            first += used[b]
            self.table[b, :used[b]] = mine.to(I32)
            t = torch.arange(n)
            self.slots.append((mine[t // M.PAGE] * M.PAGE + t % M.PAGE).to(I32))
        self.k = [torch.randn((n, self.hkv, d), generator=g) * keys for _, n in self.seqs]
        self.v = [torch.randn((n, self.hkv, d), generator=g) for _, n in self.seqs]
        self.cache = cache.cuda()
        self.write()
        offsets = [0]
        for m, _ in self.seqs:
            offsets.append(offsets[-1] + m)
        self.offsets, self.n = offsets, offsets[-1]
        self.q = torch.randn((self.n + 3, self.hq, d), generator=g).to(self.dt)
        self.scale = 1.3 * d ** -0.5
        # (three rows behind the last sequence count as rows)
        p = M.plan(dtype, self.n + 3, len(self.seqs), self.hq, self.hkv, d, width * M.PAGE)
        assert p.tiles == 0 and (p.target == 0) == M.CALLS[name][4]
        self.ws = torch.empty(lk.LOOKME_ATTENTION_WORKSPACE, dtype=torch.uint8, device="cuda")
        self.args = [torch.tensor([n for _, n in self.seqs], dtype=I32).cuda(),
                     torch.tensor(offsets, dtype=I32).cuda()]

    def write(self):
        lk.cache_write(torch.cat(self.k).cuda(), torch.cat(self.v).cuda(),
                       torch.cat(self.slots).cuda(), self.cache)

    def run(self, causal, q=None, out=None):
        q = self.q.cuda() if q is None else q
        out = torch.full_like(q, 7.0) if out is None else out
        lk.cache_attention(q, self.cache, self.table.cuda(), self.args[0], out, self.ws,
                           q_offsets=self.args[1], scale=self.scale, causal=causal)
        return out

    def rows(self, b):
        return slice(self.offsets[b], self.offsets[b + 1])

    def check(self, out, causal, keep=None):
        assert (out[self.n:] == 7).all()               # rows behind the last sequence
        for b in range(len(self.seqs)):
            at = self.rows(b)
            _close(out[at], M.attention(self.q[at], A.value(*A.quantize(self.k[b])),
                                        A.value(*A.quantize(self.v[b])), self.scale, causal,
                                        None if keep is None else keep[b]))


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "cross"])
@pytest.mark.parametrize("dtype,d", M.MANY)
@pytest.mark.parametrize("name", list(M.CALLS))
def test_many_rows(name, dtype, d, causal):
    c = Call(name, dtype, d)
    out = c.run(causal)
    c.check(out, causal)
    for _ in range(20):
        assert torch.equal(out, c.run(causal))


@pytest.mark.parametrize("dtype,d", M.MANY)
@pytest.mark.parametrize("name", ["whole", "cut"])
def test_the_first_tiles_decide(name, dtype, d):
    """keys of the first tile of a sequence that outweigh all others, and keys of the third
    that would, were they read in their place: a tile's operands stay until every wave has
    read them"""
    c = Call(name, dtype, d, keys=0.2)
    for b, (m, n) in enumerate(c.seqs):
        if m and n > 96:
            q = c.q[c.rows(b)].double().view(m, c.hkv, -1, d).mean((0, 2))
            q = (q / q.norm(dim=-1, keepdim=True)).float()
            c.q[c.rows(b)] += (2 * q).repeat_interleave(c.hq // c.hkv, 0).to(c.dt)
            c.k[b][:32] += 12 * q
            c.k[b][64:96] += 9 * q
    c.write()
    q = c.q.cuda()
    out = c.run(False, q)
    c.check(out, False)
    for _ in range(50):
        assert torch.equal(out, c.run(False, q))


@pytest.mark.parametrize("dtype,d", M.MANY)
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("name", list(M.CALLS))
def test_blocks_that_are_not_finite_reach_only_the_rows_that_see_them(name, what, dtype, d):
    """one that the last two rows of every sequence see, in a tile that others see too, and
    one in an early tile of some sequences that all rows but the first ones see"""
    c = Call(name, dtype, d)
    good = c.run(True)
    want = [M.attention(c.q[c.rows(b)], A.value(*A.quantize(c.k[b])), A.value(*A.quantize(c.v[b])),
                        c.scale, True) for b in range(len(c.seqs))]
    hit = torch.zeros(c.n, dtype=torch.bool)
    for b, (m, n) in enumerate(c.seqs):
        for bad in [n - 2] + ([n - m + 3] if b % 3 == 0 else []):
            if m >= 8 and 0 <= bad < n:
                (c.k if what == "k" else c.v)[b][bad, 0, 33] = NAN
                hit[c.offsets[b] + max(0, bad - (n - m)):c.offsets[b + 1]] = True
    c.write()
    out = c.run(True).cpu()
    good, G = good.cpu(), c.hq // c.hkv
    assert hit.any() and not hit.all()
    assert torch.equal(out[:c.n, G:], good[:c.n, G:])                # the other key heads
    if what == "v":
        assert torch.equal(out[:c.n][~hit], good[:c.n][~hit])
    else:                  # (rows of a wave renew their maxima together)
        for b in range(len(c.seqs)):
            at = c.rows(b)
            far = (out[at].double() - want[b][0]).abs() - want[b][1]
            assert not far[~hit[at]].isnan().any() and (far[~hit[at]] <= 0).all()
    out, good = out[:c.n][hit][:, :G], good[:c.n][hit][:, :G]
    if what == "k":
        assert out.isnan().all()
    else:                              # value 33 is in the second block of 32
        assert out[..., 32:64].isnan().all()
        rest = [i for i in range(d) if not 32 <= i < 64]
        assert torch.equal(out[..., rest], good[..., rest])


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "cross"])
@pytest.mark.parametrize("garbage", [255, 120])
@pytest.mark.parametrize("dtype,d", M.MANY)
@pytest.mark.parametrize("name", list(M.CALLS))
def test_pages_out_of_range(name, dtype, d, garbage, causal):
    """the first, a middle and the last page of some sequences, and all of one's, are none"""
    c = Call(name, dtype, d, garbage=garbage)
    keep = [torch.ones(n, dtype=torch.bool) for _, n in c.seqs]
    none = [-1, c.num_pages, 2 ** 31 - 1]
    for b, (m, n) in enumerate(c.seqs):
        pages = -(-n // M.PAGE)
        lost = [[0], [pages // 2], [pages - 1], [0, 1, pages - 1], range(pages)][b % 5]
        for p in lost:
            if 0 <= p < pages:
                c.table[b, p] = none[p % 3]
                keep[b][p * M.PAGE:(p + 1) * M.PAGE] = False
    c.check(c.run(causal), causal, keep)


@pytest.mark.parametrize("dtype,d", M.MANY)
@pytest.mark.parametrize("name", ["whole, many sequences", "cut", "cut, many sequences"])
def test_captured(name, dtype, d):
    """replays with other queries, eager calls and synchronizations between them, in place"""
    c = Call(name, dtype, d)
    x = c.q.cuda()
    table = c.table.cuda()

    def call():
        lk.cache_attention(x, c.cache, table, c.args[0], x, c.ws, q_offsets=c.args[1],
                           scale=c.scale)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        q = torch.randn(c.q.shape, generator=_gen(i)).to(c.dt).cuda()
        want = c.run(True, q)
        x.copy_(q)
        graph.replay()
        assert torch.equal(x[:c.n], want[:c.n]) and torch.equal(x[c.n:], q[c.n:])
        torch.cuda.synchronize()
