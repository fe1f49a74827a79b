"""Attention over the 4-bit cache at the ends of what its inputs may hold: bytes that no
write leaves, scores at and past float32's ends, more rows than a launch of waves has."""

import pytest
import torch

from paper_2607_16305_amd import lookme as lk
from tests import attention as A
from tests import attention_many as M

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
I32 = torch.int32


def _gen(seed=0):
    return torch.Generator().manual_seed(seed)


def _close(got, want):
    v, e = want
    far = (got.cpu().double() - v).abs() - e
    assert not far.isnan().any() and far.max() <= 0, f"{far.max()} past the bound"


# rows, tokens, q heads, key heads, width of the table: each kernel, whole and cut
SHAPES = {"one tile": (3, 90, 4, 2, 3), "one tile, cut": (3, 700, 4, 2, 200),
          "two tiles": (12, 90, 4, 2, 3), "two tiles, cut": (12, 700, 4, 2, 200),
          "three tiles": (22, 90, 4, 2, 3), "many, cut": (130, 400, 4, 2, 200),
          "many": (520, 90, 64, 16, 3)}
KINDS = [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 128), ("f32", 256)]


def _inputs(shape, dtype, d, seed=0):
    """(q, k, v, cache, table) of one sequence; a page that no token uses is page 0"""
    m, n, hq, hkv, width = SHAPES[shape]
    plan = M.plan(dtype, m, 1, hq, hkv, d, 32 * width)
    assert (plan.target > 0) == ("cut" in shape)
    assert (plan.tiles == 0) == ("many" in shape and (dtype, d) in M.MANY)
    g = _gen(seed)
    pages = -(-n // 32)
    q = torch.randn((m, hq, d), generator=g).to(DT[dtype])
    k, v = torch.randn((n, hkv, d), generator=g), torch.randn((n, hkv, d), generator=g)
    table = torch.full((1, width), -7, dtype=I32)
    table[0, :pages] = torch.randperm(pages, generator=g).to(I32) + 1
    cache = torch.full(lk.cache_shape(pages + 1, hkv, 32, d), 255, dtype=torch.uint8)
    return q, k, v, cache.cuda(), table


def _fill(cache, table, k, v):
    t = torch.arange(k.shape[0])
    slots = (table[0, t // 32] * 32 + t % 32).to(I32).cuda()
    lk.cache_write(k.cuda(), v.cuda(), slots, cache)


def _run(q, cache, table, n, causal, scale):
    out = torch.full_like(q, 7.0).cuda()
    ws = torch.empty(lk.LOOKME_ATTENTION_WORKSPACE, dtype=torch.uint8, device="cuda")
    lk.cache_attention(q.cuda(), cache, table.cuda(), torch.tensor([n], dtype=I32).cuda(), out, ws,
                       q_offsets=torch.tensor([0, q.shape[0]], dtype=I32).cuda(), causal=causal,
                       scale=scale)
    return out


def _values(x):
    return A.value(*A.quantize(x))


@pytest.mark.parametrize("byte", [253, 254])
@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("shape", list(SHAPES))
def test_bytes_that_no_write_leaves_in_what_a_row_does_not_see(shape, dtype, d, byte):
    """scales past the largest, 4 or 6 times which bf16 cannot hold: in the last token's v,
    which only the last row sees, and on a page 0 that the table's bad entries must not lead
    to"""
    q, k, v, cache, table = _inputs(shape, dtype, d)
    n, scale = k.shape[0], d ** -0.5
    _fill(cache, table, k, v)
    cache[0] = 0x77                                       # codes of 6
    cache[0, ..., 32 * d:] = byte
    keep = torch.ones(n, dtype=torch.bool)
    table[0, 1], keep[32:64] = -1, False
    kd, vd = _values(k), _values(v)
    _close(_run(q, cache, table, n, True, scale), M.attention(q, kd, vd, scale, True, keep))
    _close(_run(q, cache, table, n, False, scale), M.attention(q, kd, vd, scale, False, keep))
    last = n - 1
    tile = cache[int(table[0, last // 32]), :, 0]
    _, codes, _, scales = A.places(last % 32, d)
    tile[:, codes.cuda()] = 0xF7                          # 6 and -6
    tile[:, scales.cuda()] = byte
    out = _run(q, cache, table, n, True, scale)
    want = M.attention(q, kd, vd, scale, True, keep)
    _close(out[:-1], (want[0][:-1], want[1][:-1]))
    assert out[-1].isnan().all()
    got = torch.zeros((1, cache.shape[1], d), device="cuda")
    slot = table[0, last // 32] * 32 + last % 32
    lk.cache_read(slot[None].to(I32).cuda(), cache, v_out=got)
    assert got.isnan().all()


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("shape", list(SHAPES))
def test_scores_at_the_largest_scales(shape, dtype, d):
    """queries so small that the scaled scores are ordinary ones again: whole powers of two,
    so that no product with a key is a float32 denormal"""
    q, k, v, cache, table = _inputs(shape, dtype, d)
    _fill(cache, table, k, v)
    for scale, to in ((2.0 ** 126, -122), (2.0 ** 120, -122), (1e30, -100)):
        small = torch.where(q < 0, -1.0, 1.0).to(q.dtype) * 2.0 ** to
        out = _run(small, cache, table, k.shape[0], True, scale)
        _close(out, M.attention(small, _values(k), _values(v), scale, True))


def _check_range(out, q, k, v, scale):
    """out of queries and keys with one element that is not zero, every row seeing every
    token, where scaled scores may pass float32: a row with one above is NaN, those below
    weigh nothing.  The scores that stay are one product each, exact but for a rounding that
    tokens of the same key share, and apart by more than a weight can bridge or alike: no
    error of theirs counts.  (The largest power of two up to which a scaled score stays, 2^126
    or more, is the library's to choose.)"""
    hkv, G = k.shape[1], q.shape[1] // k.shape[1]
    kd, vd = _values(k)[..., 0], _values(v)
    out, most = out.cpu().double(), torch.finfo(torch.float32).max
    for h in range(q.shape[1]):
        s = scale * q[:, h, :1].double() * kd[:, h // G]                # [rows, n]
        log2 = s * 1.4426950408889634
        unsure = ((s.abs() > 2.0 ** 126) & (log2.abs() <= most)).any(-1)
        over = (log2 > most).any(-1)
        p = torch.softmax(s.masked_fill(log2 < -most, -torch.inf), -1).nan_to_num(0)
        want, size = p @ vd[:, h // G], p @ vd[:, h // G].abs()
        half = A.HALF[q.dtype] * (1 + 2.0 ** -7)
        e = (half + (len(k) + 64) * A.U32) * size + half * want.abs() + 2.0 ** -126
        assert out[over, h].isnan().all()
        rest = ~over & ~unsure
        assert not ((out[:, h] - want).abs() - e)[rest].isnan().any()
        assert (((out[:, h] - want).abs() - e)[rest] <= 0).all()


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("shape", list(SHAPES))
def test_scaled_scores_past_float32(shape, dtype, d):
    """minus infinity weighs nothing, alone it gives 0; plus infinity gives NaN"""
    q, k, v, cache, table = _inputs(shape, dtype, d)
    n = k.shape[0]
    q[..., 0] = q[..., 0].abs() + 1
    q[..., 1:] = 0
    k[:, :, 0] = -k[:, :, 0].abs() - 1                    # every score is below zero
    _fill(cache, table, k, v)
    assert not _run(q * 1e20, cache, table, n, False, 1e30).any()
    huge = [(sign * top, scale) for sign in (1, -1)
            for top, scale in ((1.0, 2.0 ** 126), (1.0, 1e30), (1e20, 1e30))]
    for top, scale in huge:
        _check_range(_run(q * top, cache, table, n, False, scale), q * top, k, v, scale)
    # some tokens with scores of zero: they share the row
    k[torch.rand(n, generator=_gen(3)) < 0.4, :, 0] = 0
    _fill(cache, table, k, v)
    for top, scale in huge:
        _check_range(_run(q * top, cache, table, n, False, scale), q * top, k, v, scale)


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("shape", list(SHAPES))
def test_scores_whose_spacing_is_more_than_a_weight_can_bridge(shape, dtype, d):
    """scaled scores from 2^12 to 2^100, positive and negative: the tokens with the largest
    share the row, however its maximum is rounded"""
    q, k, v, cache, table = _inputs(shape, dtype, d)
    q[..., 0] = q[..., 0].abs() + 1
    q[..., 1:] = 0
    _fill(cache, table, k, v)
    for log2 in (12, 24, 28, 29, 30, 31, 32, 36, 45, 63, 100):
        for sign in (1.3, -1.1):
            x, scale = q * sign, 1.7 * 2.0 ** log2
            _check_range(_run(x, cache, table, k.shape[0], False, scale), x, k, v, scale)


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("shape", list(SHAPES))
def test_queries_at_and_past_the_end_of_their_type(shape, dtype, d):
    """infinite ones: a row whose scores are all minus infinity gives 0, one with plus infinity
    NaN, the others what they were; and the largest finite ones, over keys so small that the
    scores are ordinary"""
    q, k, v, cache, table = _inputs(shape, dtype, d)
    m, n, scale = q.shape[0], k.shape[0], d ** -0.5
    k[..., 3] = k[..., 3].abs() + 1
    _fill(cache, table, k, v)
    good = _run(q, cache, table, n, False, scale).cpu()
    q[0, 0, 3], q[m // 2, 1, 3], q[m - 1, -1, 3] = -torch.inf, torch.inf, -torch.inf
    out = _run(q, cache, table, n, False, scale).cpu()
    assert not out[0, 0].any() and not out[m - 1, -1].any() and out[m // 2, 1].isnan().all()
    want = M.attention(q.nan_to_num(0, 0, 0), _values(k), _values(v), scale, False)
    rest = torch.ones(q.shape[:2], dtype=torch.bool)
    rest[0, 0] = rest[m // 2, 1] = rest[m - 1, -1] = False
    assert ((out.double() - want[0]).abs() <= want[1])[rest].all()
    assert good.isfinite().all()
    # (a block of keys of 2^-98 and less, queries of nearly 2^128)
    k[..., :32] *= 2.0 ** -98
    most = torch.finfo(q.dtype).max
    q = torch.randn(q.shape, generator=_gen(8)).to(q.dtype) * 2.0 ** 10
    q[..., :32] = torch.where(torch.rand(q[..., :32].shape, generator=_gen(9)) < 0.5, most, -most)
    q[..., :4] *= 0.9990234375
    _fill(cache, table, k, v)
    scale = 2.0 ** -33
    _close(_run(q, cache, table, n, True, scale),
           M.attention(q, _values(k), _values(v), scale, True))


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("shape", list(SHAPES))
def test_the_largest_sums(shape, dtype, d):
    """values of which as many as there are tokens, times 2^8, stay below float32's end"""
    q, k, v, cache, table = _inputs(shape, dtype, d)
    n, scale = k.shape[0], d ** -0.5
    v *= 2.0 ** (119 - n.bit_length()) / 8                # (v is below 8, as is what is kept of it)
    _fill(cache, table, k, v)
    assert v.abs().max() * n < 2.0 ** 119 and _values(v).abs().max() * n < 2.0 ** 119
    for causal in (True, False):
        _close(_run(q, cache, table, n, causal, scale),
               M.attention(q, _values(k), _values(v), scale, causal))


def test_the_parts_of_more_rows_than_a_launch_are_joined():
    """2^26 rows of query heads, a wave each, of which the first and the last sequence's have
    cut keys: alike, so that the outputs are averages of small whole numbers"""
    B, heads, d, page = 1 << 17, 512, 64, 1 << 20
    plan = M.plan("bf16", B, B, heads, 1, d, 8 * page)
    assert plan.target > 0 and B * heads * 64 >= 2 ** 32
    cache = torch.zeros(lk.cache_shape(2, 1, page, d), dtype=torch.uint8, device="cuda")
    k = torch.ones((page, 1, d), dtype=torch.bfloat16, device="cuda")
    t = torch.arange(page, dtype=I32, device="cuda")
    for p in (0, 1):
        v = (t % 4 + 2 * p).to(k.dtype)[:, None, None].expand(page, 1, d).contiguous()
        lk.cache_write(k, v, t + p * page, cache)
    table = torch.zeros((B, 8), dtype=I32)
    table[-1] = 1
    lengths = torch.arange(B, dtype=I32) % 5
    want = torch.tensor([0, 0, 0.5, 1.0, 1.5])[lengths.long()]
    lengths[0] = lengths[-1] = 8 * page
    held = _values((torch.arange(8) % 4 + torch.arange(8) // 4 * 2).float()[:, None].expand(8, 32))
    assert held[:, 0].tolist() == [0, 1, 2, 3, 2, 3, 4, 4]      # (5 is as near to 4 as to 6)
    want[0], want[-1] = held[:4].mean(), held[4:].mean()
    x = torch.full((B, heads, d), 0.25, dtype=k.dtype, device="cuda")
    ws = torch.empty(lk.LOOKME_ATTENTION_WORKSPACE, dtype=torch.uint8, device="cuda")
    lk.cache_attention(x, cache, table.cuda(), lengths.cuda(), x, ws)
    for part, w in zip(x.view(B, -1).split(4096), want.split(4096)):
        assert torch.equal(part.amin(1).float().cpu(), w)
        assert torch.equal(part.amax(1).float().cpu(), w)
    # (the kernel did cut them: what it leaves for the join)
    blocks = 2 * plan.target * plan.block * (d + 2) * 4
    assert ws[blocks:blocks + 4].view(I32).item() == 1
