"""The operators of an attention sublayer on the GPU against plain float64 forms:
head norms with rotary positions, the 4-bit cache, attention over it."""

import math

import pytest
import torch

from paper_2607_16305_amd import lookme as lk
from tests import attention as A

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
I32 = torch.int32
NAN, INF = float("nan"), float("inf")


def _gen(seed=0):
    return torch.Generator().manual_seed(seed)


def _close(got, want):
    v, e = want
    far = (got.cpu().double() - v).abs() - e
    assert not far.isnan().any() and far.max() <= 0, f"{far.max()} past the bound"


# ---- head norms and positions ------------------------------------------------------

ROTARY = [
    # n, q heads, k heads, d, rot, interleaved, axes, norm, farthest position
    (1, 16, 2, 128, 128, False, 1, True, 4096),
    (1, 1, 0, 64, 0, False, 1, True, 1),
    (5, 3, 1, 128, 128, True, 1, True, 10 ** 6),
    (37, 8, 2, 256, 64, False, 3, False, 2 ** 31 - 64),
    (64, 6, 2, 80, 40, True, 3, True, 10 ** 6),
    (130, 5, 5, 72, 36, False, 2, True, 50000),        # pairs that lie across chunks
    (33, 2, 1, 8, 6, False, 1, True, 1000),
    (700, 32, 8, 64, 64, False, 1, False, 131072),
    (2100, 12, 4, 128, 128, False, 3, True, 32768),    # several tokens a workgroup
    (3000, 20, 4, 256, 2, True, 1, True, 10 ** 6),
    (2500, 9, 3, 136, 0, False, 1, True, 1),
]


def _rotary_inputs(dt, n, hq, hk, d, rot, axes, far, seed=0):
    g = _gen(seed)
    packed = (2 * torch.randn((n, hq + 2 * hk, d), generator=g)).to(dt)
    weights = [(1 + 0.2 * torch.randn(d, generator=g)).to(dt) for _ in range(2)]
    pos = torch.randint(-5, far, (axes, n), generator=g, dtype=torch.int64).to(I32)
    half = rot // 2
    freq = torch.tensor([1e6 ** (-i / max(1, half)) for i in range(half)], dtype=torch.float32)
    axis = torch.arange(half, dtype=I32) % axes if axes > 1 else None
    return packed, weights, pos if axes > 1 else pos[0], freq, axis


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("case", ROTARY, ids=str)
def test_head_norm_rotary(dtype, case):
    n, hq, hk, d, rot, inter, axes, norm, far = case
    dt = DT[dtype]
    packed, weights, pos, freq, axis = _rotary_inputs(dt, n, hq, hk, d, rot, axes, far)
    x = packed.cuda()
    outs = [torch.full((n, h + 1, d), 7.0, dtype=dt, device="cuda") for h in (hq, hk)]
    q_out, k_out = outs[0][:, :hq], outs[1][:, :hk]          # rows that lie apart
    on = lambda t: None if t is None else t.cuda()  # noqa: E731
    kw = dict(eps=1e-5, norm=norm, factor=1.25, interleaved=inter)
    if rot:
        kw.update(pos=on(pos), freq=on(freq), axis=on(axis))
    if hk:
        kw.update(k=x[:, hq:hq + hk], k_out=k_out)
    if norm:
        kw.update(q_weight=on(weights[0]))     # (k without a weight)
    lk.head_norm_rotary(x[:, :hq], q_out, **kw)
    plain = dict(eps=1e-5 if norm else None, pos=pos, freq=freq if rot else None, axis=axis,
                 factor=1.25, interleaved=inter)
    _close(q_out, A.rotary(packed[:, :hq], weight=weights[0] if norm else None, **plain))
    if hk:
        _close(k_out, A.rotary(packed[:, hq:hq + hk], **plain))
    assert (outs[0][:, hq:] == 7).all() and (outs[1][:, hk:] == 7).all()


@pytest.mark.parametrize("dtype", list(DT))
def test_head_norm_rotary_in_place(dtype):
    dt = DT[dtype]
    packed, weights, pos, freq, axis = _rotary_inputs(dt, 300, 6, 2, 128, 96, 1, 5000)
    x = packed.cuda()
    w = [t.cuda() for t in weights]
    lk.head_norm_rotary(x[:, :6], x[:, :6], k=x[:, 6:8], k_out=x[:, 6:8], q_weight=w[0],
                        k_weight=w[1], pos=pos.cuda(), freq=freq.cuda())
    plain = dict(eps=1e-6, pos=pos, freq=freq)
    _close(x[:, :6], A.rotary(packed[:, :6], weight=weights[0], **plain))
    _close(x[:, 6:8], A.rotary(packed[:, 6:8], weight=weights[1], **plain))
    assert torch.equal(x[:, 8:].cpu(), packed[:, 8:])


def test_head_norm_rotary_of_rows_of_zeros_infinities_and_axes_out_of_range():
    x = torch.randn((4, 2, 64), generator=_gen()).cuda()
    x[0, 0] = 0
    x[1, 0, 5] = NAN
    x[2, 1, 7] = INF
    out = torch.empty_like(x)
    freq = torch.rand(32, generator=_gen(1))
    pos = torch.randint(0, 99, (2, 4), generator=_gen(2), dtype=I32)
    axis = torch.arange(32, dtype=I32) - 10          # clamped to 0 and 1
    lk.head_norm_rotary(x, out, pos=pos.cuda(), freq=freq.cuda(), axis=axis.cuda())
    want, e = A.rotary(x.cpu(), eps=1e-6, pos=pos, freq=freq, axis=axis.clamp(0, 1))
    bad = torch.zeros(4, 2, dtype=torch.bool)
    bad[1, 0] = bad[2, 1] = True
    assert ((out.cpu().double() - want).abs() <= e)[~bad].all()
    assert not out[0, 0].any() and out[1, 0].isnan().all() and out[2, 1, 7].isnan()


# ---- the cache -------------------------------------------------------------------------

def _awkward(shape, dt, seed=0):
    """values at and beside the rounding's borders, blocks of zeros, tiny and huge
    ones, with infinities and NaN"""
    g = _gen(seed)
    x = torch.randn(shape, generator=g)
    x = x * torch.exp2(torch.randint(-6, 7, shape[:2] + (1,), generator=g).float())
    flat = x.view(-1, 32)
    rows = flat.shape[0]
    border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0])
    flat[0::7, :9] = border
    flat[0::7, 9:] = (flat[0::7, 9:] % 1).abs() * -4
    if dt is torch.float32:
        flat[3::7, :9] = torch.nextafter(border, torch.tensor(9.0))
        flat[4::7, 9:18] = -torch.nextafter(border, torch.tensor(0.0))
    flat[1::11] = 0
    flat[2::13] *= 2.0 ** -110
    flat[4::17] *= 2.0 ** 119
    flat[5::19, 3] = -0.0
    if rows > 40:
        flat[23, 7], flat[29, 31], flat[31, 0] = INF, NAN, -INF
        flat[37] = 3e38
    return x.to(dt)


CACHE = [(1, 1, 64, 32), (5, 2, 128, 32), (64, 8, 128, 64), (70, 3, 256, 128), (333, 2, 64, 256),
         (1000, 4, 128, 1024), (129, 1, 256, 32)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n,heads,d,page", CACHE)
def test_cache_write_and_read(dtype, n, heads, d, page):
    dt, g = DT[dtype], _gen(n)
    pages = -(-n // page) + 1
    k, v = _awkward((n, heads, d), dt), _awkward((n, heads, d), dt, 1)
    slots = torch.randperm(pages * page, generator=g)[:n].to(I32)
    if n > 4:
        slots[2], slots[3], slots[4] = -1, pages * page, 2 ** 31 - 1
    before = torch.randint(0, 256, lk.cache_shape(pages, heads, page, d), generator=g,
                           dtype=torch.uint8)
    cache = before.cuda()
    both = torch.cat([k, v, k], 1).cuda()            # rows that lie apart
    lk.cache_write(both[:, :heads], both[:, heads:2 * heads], slots.cuda(), cache)
    want = A.write(before, slots, k, v)
    assert torch.equal(cache.cpu(), want)
    live = (slots >= 0) & (slots < pages * page)
    wk, wv = A.read(want, slots[live])
    for out_dt in DT.values():
        out = torch.full((n, 2 * heads, d), 7.0, dtype=out_dt, device="cuda")
        lk.cache_read(slots.cuda(), cache, out[:, :heads], out[:, heads:])
        got = out.cpu().double()
        for x, w in ((got[:, :heads], wk), (got[:, heads:], wv)):
            assert torch.equal(x[live].nan_to_num(12345.0), w.nan_to_num(12345.0))
            assert (x[~live] == 7).all()
        one = torch.full((n, heads, d), 7.0, dtype=out_dt, device="cuda")
        lk.cache_read(slots.cuda(), cache, v_out=one)
        assert torch.equal(one.cpu().double().nan_to_num(12345.0),
                           got[:, heads:].nan_to_num(12345.0))
        lk.cache_read(slots.cuda(), cache, k_out=one)
        assert torch.equal(one.cpu().double().nan_to_num(12345.0),
                           got[:, :heads].nan_to_num(12345.0))


def test_cache_rows_do_not_depend_on_their_batch():
    g = _gen(3)
    k, v = torch.randn((96, 2, 128), generator=g).cuda(), torch.randn((96, 2, 128), generator=g).cuda()
    slots = torch.arange(96, dtype=I32).cuda()
    all_at_once = torch.zeros(lk.cache_shape(3, 2, 32, 128), dtype=torch.uint8, device="cuda")
    one_by_one = torch.zeros_like(all_at_once)
    lk.cache_write(k, v, slots, all_at_once)
    for i in range(96):
        lk.cache_write(k[i:i + 1], v[i:i + 1], slots[i:i + 1].clone(), one_by_one)   # (16-byte aligned)
    assert torch.equal(all_at_once, one_by_one)


# ---- attention --------------------------------------------------------------------------

def _sequences(seqs, hkv, d, page, seed=0, garbage=255):
    """A cache with the sequences' k and v (of their lengths), what lies behind them
    `garbage`, the page table, and the values it holds"""
    g = _gen(seed)
    width = max(1, max(-(-n // page) for _, n in seqs))
    used = [-(-n // page) for _, n in seqs]
    pages = sum(used) + 2
    order = torch.randperm(pages, generator=g)
    table = torch.full((len(seqs), width), -7, dtype=I32)    # (behind a length: not read)
    cache = torch.full(lk.cache_shape(pages, hkv, page, d), garbage, dtype=torch.uint8)
    k = [(torch.randn((n, hkv, d), generator=g) * 1.5) for _, n in seqs]
    v = [torch.randn((n, hkv, d), generator=g) for _, n in seqs]
    first, slots = 0, []
    for b, (_, n) in enumerate(seqs):
        mine = order[first:first + used[b]]
        first += used[b]
        table[b, :used[b]] = mine.to(I32)
        t = torch.arange(n)
        slots.append(mine[t // page] * page + t % page)
    slots = torch.cat(slots).to(I32)
    cache = cache.cuda()
    lk.cache_write(torch.cat(k).cuda(), torch.cat(v).cuda(), slots.cuda(), cache)
    vals = []
    for a, b in zip(k, v):
        vals.append((A.value(*A.quantize(a)), A.value(*A.quantize(b))))
    return cache, table, slots, vals


def _run(q, cache, table, seqs, causal=True, scale=None, offsets=True, out=None, **kw):
    off = [0]
    for m, _ in seqs:
        off.append(off[-1] + m)
    out = torch.full_like(q, 7.0) if out is None else out
    ws = torch.empty(lk.LOOKME_ATTENTION_WORKSPACE, dtype=torch.uint8, device="cuda")
    lk.cache_attention(q, cache, table.cuda(), torch.tensor([n for _, n in seqs], dtype=I32).cuda(),
                       out, ws, q_offsets=torch.tensor(off, dtype=I32).cuda() if offsets else None,
                       causal=causal, scale=scale, **kw)
    return out


def _check(out, q, vals, seqs, causal, scale):
    a = 0
    for (m, _), (k, v) in zip(seqs, vals):
        if m:
            _close(out[a:a + m], A.attention(q[a:a + m], k, v, scale, causal))
        a += m


ATTENTION = [
    # (rows, length) of the sequences, q heads, kv heads, page
    ([(1, 1)], 1, 1, 32), ([(1, 31)], 4, 1, 32), ([(1, 33)], 8, 2, 32), ([(1, 700)], 6, 2, 64),
    ([(1, 5), (1, 0), (1, 300), (1, 64), (1, 1000)], 8, 2, 64),
    ([(1, n) for n in range(1, 131, 2)], 4, 4, 32),              # more sequences than lanes
    ([(5, 200), (3, 3), (1, 90), (0, 50), (7, 4), (2, 1)], 6, 2, 32),   # rows that see nothing
    ([(17, 129)], 7, 1, 128), ([(40, 300), (130, 131)], 4, 2, 64),
    ([(1, 6000)], 16, 2, 256), ([(3, 2500), (2, 90)], 40, 2, 32),   # over 16 rows, keys cut
    ([(260, 777)], 3, 1, 1024),
]


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "cross"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("case", ATTENTION, ids=[str(i) for i in range(len(ATTENTION))])
def test_cache_attention(case, dtype, d, causal):
    seqs, hq, hkv, page = case
    cache, table, _, vals = _sequences(seqs, hkv, d, page)
    n = sum(m for m, _ in seqs)
    q = torch.randn((n + 3, hq, d), generator=_gen(5)).to(DT[dtype])
    scale = 1.3 * d ** -0.5
    out = _run(q.cuda(), cache, table, seqs, causal, scale)
    assert (out[n:] == 7).all()                        # rows behind the last sequence
    _check(out[:n], q, vals, seqs, causal, scale)
    again = _run(q.cuda(), cache, table, seqs, causal, scale)
    assert torch.equal(out, again)


@pytest.mark.parametrize("wide", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("m", [5, 12, 23, 31, 45, 70])
def test_cache_attention_of_every_count_of_rows(m, dtype, d, wide):
    """10 to 140 rows a key head, the keys whole and (a table that could hold more) cut"""
    seqs = [(m, 500), (m + 1, 190), (m - 4, 31), (m, m)]
    cache, table, _, vals = _sequences(seqs, 2, d, 32)
    if wide:
        table = torch.cat([table, torch.full((4, 2000), -7, dtype=I32)], 1)
    n = sum(r for r, _ in seqs)
    need = lk.lookme_cache_attention_workspace(int(dtype == "bf16"), n, 4, 4, 2, d,
                                               table.shape[1], 32)
    assert need > 0 or not wide
    q = torch.randn((n, 4, d), generator=_gen(m)).to(DT[dtype])
    for causal in (True, False):
        out = _run(q.cuda(), cache, table, seqs, causal)
        _check(out, q, vals, seqs, causal, d ** -0.5)


@pytest.mark.parametrize("seqs,hq,hkv", [
    ([(1, 5000)] + [(1, 37)] * 130, 8, 8),    # one long sequence among short ones: cut
    ([(300, 320), (290, 290)], 16, 1),        # rows enough and few tokens: whole
])
@pytest.mark.parametrize("d", [64, 128])
def test_the_lengths_choose_whether_keys_are_cut(seqs, hq, hkv, d):
    cache, table, _, vals = _sequences(seqs, hkv, d, 32)
    table = torch.cat([table, torch.full((len(seqs), 8000), -7, dtype=I32)], 1)
    n = sum(r for r, _ in seqs)
    assert lk.lookme_cache_attention_workspace(1, n, len(seqs), hq, hkv, d, table.shape[1], 32) > 0
    q = torch.randn((n, hq, d), generator=_gen(n)).bfloat16()
    out = _run(q.cuda(), cache, table, seqs)
    _check(out, q, vals, seqs, True, d ** -0.5)
    assert torch.equal(out, _run(q.cuda(), cache, table, seqs))


@pytest.mark.parametrize("wide", [False, True], ids=["narrow", "wide"])
@pytest.mark.parametrize("hq,hkv", [(14, 2), (4, 4), (12, 1)])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "bf16"), (256, "f32")])
def test_many_sequences(d, dtype, hq, hkv, wide):
    """more sequences than a wave has lanes: without rows, without tokens, and a long one"""
    g = _gen(hq)
    rows = torch.tensor([0, 1, 1, 2, 5, 11])[torch.randint(0, 6, (90,), generator=g)].tolist()
    lens = torch.randint(0, 150, (90,), generator=g).tolist()
    rows[-3:], lens[70] = [0, 3, 0], 1800
    seqs = list(zip(rows, lens))
    cache, table, _, vals = _sequences(seqs, hkv, d, 32)
    if wide:
        table = torch.cat([table, torch.full((90, 9000), -7, dtype=I32)], 1)
    n = sum(rows)
    q = torch.randn((n + 40, hq, d), generator=g).to(DT[dtype])
    out = _run(q.cuda(), cache, table, seqs)
    assert (out[n:] == 7).all()
    _check(out[:n], q, vals, seqs, True, d ** -0.5)


def test_rows_apart_in_place_and_without_offsets():
    seqs = [(1, 77), (1, 1200), (1, 0)]
    cache, table, _, vals = _sequences(seqs, 2, 128, 64)
    packed = torch.randn((3, 12, 128), generator=_gen(1)).bfloat16()
    x = packed.cuda()
    out = _run(x[:, 2:10], cache, table, seqs, offsets=False, out=x[:, 2:10])
    assert out.data_ptr() == x[:, 2:10].data_ptr()
    _check(x[:, 2:10], packed[:, 2:10].contiguous(), vals, seqs, True, 128 ** -0.5)
    assert not x[2, 2:10].any()
    assert torch.equal(x[:, :2].cpu(), packed[:, :2]) and torch.equal(x[:, 10:].cpu(), packed[:, 10:])


@pytest.mark.parametrize("dtype", list(DT))
def test_large_scores_and_one_token_that_wins(dtype):
    """scores in the thousands: the running maximum moves far and often"""
    seqs = [(2, 900), (20, 400)]
    cache, table, _, vals = _sequences(seqs, 1, 128, 64)
    q = (300 * torch.randn((22, 2, 128), generator=_gen(2))).to(DT[dtype])
    out = _run(q.cuda(), cache, table, seqs, True, 1.0)
    _check(out, q, vals, seqs, True, 1.0)


def _with(cache, slots, rows, what, heads=None):
    """the same cache with k or v of some rows (of the slots) not finite, by a write"""
    pages, hkv, tiles, width = cache.shape
    d = width // 34
    k, v = torch.empty((len(rows), hkv, d)).cuda(), torch.empty((len(rows), hkv, d)).cuda()
    at = slots[rows].cuda()
    lk.cache_read(at, cache, k, v)
    (k if what == "k" else v)[:, 0, 33] = NAN
    lk.cache_write(k, v, at, cache)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("m", [3, 11, 20, 30, 60])
def test_blocks_that_are_not_finite_reach_only_the_rows_that_see_them(what, m, d):
    n = 200
    seqs = [(m, n)]
    cache, table, slots, vals = _sequences(seqs, 2, d, 32)
    q = torch.randn((m, 4, d), generator=_gen(7)).bfloat16()
    good = _run(q.cuda(), cache, table, seqs)
    bad = n - 2                        # seen by the last two rows
    _with(cache, slots, [bad], what)
    out = _run(q.cuda(), cache, table, seqs)
    first = m - 2
    assert torch.equal(out[:first], good[:first])
    assert torch.equal(out[:, 2:], good[:, 2:])                       # the other key head
    hit = out[first:, :2].cpu()
    if what == "k":
        assert hit.isnan().all()
    else:                              # value 33 is in the second block of 32
        assert hit[..., 32:64].isnan().all()
        rest = [i for i in range(d) if not 32 <= i < 64]
        assert torch.equal(hit[..., rest], good[first:, :2].cpu()[..., rest])
    # a query that is not finite reaches its own row and head
    q2 = q.clone()
    q2[0, 1, 9] = NAN
    out2 = _run(q2.cuda(), cache, table, seqs)
    assert out2[0, 1].isnan().all()
    same = torch.ones(m, 4, dtype=torch.bool)
    same[0, 1] = False
    assert torch.equal(out2.cpu()[same].nan_to_num(9e9), out.cpu()[same].nan_to_num(9e9))


def test_pages_and_lengths_out_of_range():
    """a page that is none leaves its tokens out; lengths and offsets are clamped"""
    seqs = [(1, 300), (1, 64)]
    cache, table, _, vals = _sequences(seqs, 2, 64, 32)
    q = torch.randn((2, 4, 64), generator=_gen(3))
    table[0, 2], table[0, 5], table[0, 9] = -1, cache.shape[0], 2 ** 31 - 1
    out = _run(q.cuda(), cache, table, seqs)
    keep = torch.tensor([t for t in range(300) if t // 32 not in (2, 5, 9)])
    k, v = vals[0]
    _close(out[:1], A.attention(q[:1], k[keep], v[keep], 0.125, False))
    _close(out[1:], A.attention(q[1:], *vals[1], 0.125, True))
    none = torch.full_like(table, -1)
    assert not _run(q.cuda(), cache, none, seqs).any()
    # lengths past the table's width are its width, below zero are zero
    table = torch.zeros((2, 2), dtype=I32)
    out = torch.full_like(q, 7.0).cuda()
    ws = torch.empty(lk.LOOKME_ATTENTION_WORKSPACE, dtype=torch.uint8, device="cuda")
    cache.zero_()
    v1 = torch.ones((64, 2, 64))
    lk.cache_write(v1.cuda(), v1.cuda(), torch.arange(64, dtype=I32).cuda(), cache)
    lk.cache_attention(q.cuda(), cache, table.cuda(),
                       torch.tensor([2 ** 31 - 1, -5], dtype=I32).cuda(), out, ws)
    assert (out[0] - 1).abs().max() < 2.0 ** -20 and not out[1].any()
    out.fill_(7.0)
    lk.cache_attention(q.cuda(), cache, table.cuda(), torch.tensor([9, 9], dtype=I32).cuda(), out,
                       ws, q_offsets=torch.tensor([-4, 1, 2 ** 30], dtype=I32).cuda())
    assert (out - 1).abs().max() < 2.0 ** -20
    out.fill_(7.0)
    lk.cache_attention(q.cuda(), cache, table.cuda(), torch.tensor([9, 9], dtype=I32).cuda(), out,
                       ws, q_offsets=torch.tensor([0, 0, 1], dtype=I32).cuda())
    assert (out[0] - 1).abs().max() < 2.0 ** -20 and (out[1] == 7).all()


def test_exact_averages():
    """keys alike give every token the same weight: averages of small whole numbers,
    exact in float32, whatever cuts the keys"""
    for n in (1, 2, 32, 64, 4096, 65536):
        m = 1
        k = torch.ones((n, 1, 128))
        v = (torch.arange(n) % 4).float()[:, None, None].expand(n, 1, 128).contiguous()
        cache = torch.zeros(lk.cache_shape(-(-n // 64), 1, 64, 128), dtype=torch.uint8).cuda()
        lk.cache_write(k.cuda(), v.cuda(), torch.arange(n, dtype=I32).cuda(), cache)
        q = torch.ones((m, 1, 128))
        table = torch.arange(-(-n // 64), dtype=I32)[None]
        for dt in DT.values():
            out = _run(q.to(dt).cuda(), cache, table, [(1, n)])
            want = v.double().mean()
            assert (out.double().cpu() - want).abs().max() <= A.HALF[dt] * want


@pytest.mark.parametrize("wide", [0, 600])
@pytest.mark.parametrize("batch", [32, 80])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("m", [3, 20, 200])
def test_sequences_that_share_rows_stay_in_their_memory(m, d, batch, wide):
    """offsets that are not ascending: what such rows get is not specified, the rest of
    the outputs and of the workspace is left as it was"""
    cache = torch.full(lk.cache_shape(40, 2, 64, d), 120, dtype=torch.uint8, device="cuda")
    table = torch.randint(0, 40, (batch, 11 + wide), generator=_gen(m), dtype=I32)
    q = torch.randn((m + 3, 8, d), generator=_gen(4)).bfloat16().cuda()
    off = torch.tensor([0, m] * (batch // 2) + [m + 1], dtype=I32).cuda()   # (the last: its own)
    lens = torch.full((batch,), 700, dtype=I32).cuda()
    need = lk.lookme_cache_attention_workspace(1, m + 3, batch, 8, 2, d, table.shape[1], 64)
    for fill in (0, 255, 1):              # (what an earlier call may have left in the workspace)
        out = torch.full_like(q, 7.0)
        ws = torch.full((need + 4096,), fill, dtype=torch.uint8, device="cuda")
        lk.cache_attention(q, cache, table.cuda(), lens, out, ws[:need] if need else ws,
                           q_offsets=off)
        assert (out[m + 1:] == 7).all() and (ws[need:] == fill).all()


def test_smallest_and_largest_scales():
    """a score's range that float32 can hold: weights that are all alike, or one"""
    seqs = [(2, 400)]
    cache, table, slots, vals = _sequences(seqs, 1, 128, 32)
    table[0, 0] = -1                      # (its tokens are left out: a first tile of nothing)
    q = torch.randn((2, 1, 128), generator=_gen(6)).bfloat16()
    k, v = vals[0]
    for scale in (1e-44, 1e-38, 1e-30, 1e4):
        out = _run(q.cuda(), cache, table, seqs, False, scale)
        _check(out, q, [(k[32:], v[32:])], seqs, False, scale)
