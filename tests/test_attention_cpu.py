"""The operators of an attention sublayer without a GPU: argument checks of their
entry points before anything is launched (stand-in device addresses, never
dereferenced), the checks of the torch bindings, and the plain forms that the GPU
tests compare with."""

import math

import pytest
import torch

from paper_2607_16305_amd import lookme as lk
from tests import attention as A

P = 0x7F0000100000     # an aligned stand-in address
OK, INVALID, UNSUPPORTED = lk.LOOKME_OK, lk.LOOKME_ERR_INVALID, lk.LOOKME_ERR_UNSUPPORTED
WORKSPACE = lk.LOOKME_ERR_WORKSPACE
BF, F32 = lk.LOOKME_BF16, lk.LOOKME_F32
INF, NAN = float("inf"), float("nan")


def _status(fn, *a, **kw):
    try:
        fn(*a, **kw)
    except lk.LookmeError as e:
        assert str(e)
        return e.status
    return OK


ROTARY = dict(dtype=BF, n=4, head_dim=64, q_heads=4, q=P, q_stride=256, q_out=P, q_out_stride=256,
              k_heads=2, k=P, k_stride=256, k_out=P, k_out_stride=256, norm=1, q_weight=P,
              k_weight=None, eps=1e-6, rot=64, interleaved=0, axes=1, pos=P, axis=None, freq=P,
              factor=1.0)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), INVALID), (dict(n=-1), INVALID), (dict(n=2 ** 30 + 1), UNSUPPORTED),
    (dict(head_dim=0), INVALID), (dict(head_dim=60), UNSUPPORTED),
    (dict(dtype=F32, head_dim=6), UNSUPPORTED),
    (dict(head_dim=264, q_stride=2 ** 12, q_out_stride=2 ** 12, k_stride=2 ** 12,
          k_out_stride=2 ** 12), UNSUPPORTED),
    (dict(q_heads=0), INVALID), (dict(q_heads=4097), UNSUPPORTED), (dict(k_heads=-1), INVALID),
    (dict(q_stride=255), INVALID), (dict(q_stride=260, q=P + 16), UNSUPPORTED),
    (dict(q_out_stride=2 ** 31 + 8), UNSUPPORTED), (dict(k_stride=120), INVALID),
    (dict(k_out_stride=-8), INVALID), (dict(norm=2), INVALID), (dict(norm=0), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=NAN), INVALID), (dict(rot=66), INVALID),
    (dict(rot=31), INVALID), (dict(rot=-2), INVALID), (dict(interleaved=2), INVALID),
    (dict(rot=0), INVALID), (dict(axes=0), INVALID), (dict(factor=INF), INVALID),
    (dict(factor=NAN), INVALID), (dict(q=None), INVALID), (dict(q_out=P + 8), INVALID),
    (dict(k=None), INVALID), (dict(k_out=None), INVALID), (dict(q_out_stride=512), INVALID),
    (dict(k_out_stride=512), INVALID), (dict(q_weight=P + 2), INVALID),
    (dict(k_weight=P + 4), INVALID), (dict(pos=None), INVALID), (dict(axis=P + 4), INVALID),
    (dict(freq=None), INVALID),
    (dict(n=0, q=None, q_out=None, k=None, k_out=None, pos=None, freq=None), OK)])
def test_head_norm_rotary_refuses(kw, status):
    a = dict(ROTARY)
    a.update(kw)
    assert _status(lk.lookme_head_norm_rotary, *a.values(), 0) == status


CACHE = [
    (dict(dtype=2), INVALID), (dict(n=-1), INVALID), (dict(n=2 ** 30 + 1), UNSUPPORTED),
    (dict(kv_heads=0), INVALID), (dict(kv_heads=4097), UNSUPPORTED), (dict(head_dim=0), INVALID),
    (dict(head_dim=96), UNSUPPORTED), (dict(page=0), INVALID), (dict(page=16), UNSUPPORTED),
    (dict(page=96), UNSUPPORTED), (dict(page=2 ** 21), UNSUPPORTED), (dict(pages=0), INVALID),
    (dict(pages=2 ** 26 + 1), UNSUPPORTED), (dict(k_stride=128), INVALID),
    (dict(v_stride=260), UNSUPPORTED), (dict(slots=None), INVALID), (dict(slots=P + 4), INVALID),
    (dict(cache=None), INVALID), (dict(cache=P + 8), INVALID), (dict(k=P + 2), INVALID),
    (dict(v=P + 8), INVALID), (dict(n=0, slots=None, cache=None, k=None, v=None), OK)]


@pytest.mark.parametrize("kw,status", CACHE + [(dict(k=None), INVALID), (dict(v=None), INVALID)])
def test_cache_write_refuses(kw, status):
    a = dict(dtype=BF, n=5, kv_heads=2, head_dim=128, k=P, k_stride=256, v=P, v_stride=256, slots=P,
             pages=8, page=32, cache=P)
    a.update(kw)
    assert _status(lk.lookme_cache_write, *a.values(), 0) == status


@pytest.mark.parametrize("kw,status", CACHE + [(dict(k=None, v=None), INVALID)])
def test_cache_read_refuses(kw, status):
    a = dict(dtype=BF, n=5, kv_heads=2, head_dim=128, slots=P, pages=8, page=32, cache=P, k=P,
             k_stride=256, v=P, v_stride=256)
    a.update(kw)
    assert _status(lk.lookme_cache_read, *a.values(), 0) == status


ATTENTION = dict(dtype=BF, n=6, batch=2, q_heads=4, kv_heads=2, head_dim=128, q=P, q_stride=512,
                 q_offsets=P, lengths=P, pages=P, max_pages=3, num_pages=8, page=64, cache=P,
                 scale=0.1, causal=1, out=P, out_stride=512, workspace=P,
                 workspace_bytes=lk.LOOKME_ATTENTION_WORKSPACE)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), INVALID), (dict(n=-1), INVALID), (dict(n=2 ** 25 + 1), UNSUPPORTED),
    (dict(batch=-1), INVALID), (dict(batch=2 ** 22), UNSUPPORTED), (dict(q_heads=0), INVALID),
    (dict(kv_heads=0), INVALID), (dict(q_heads=5, q_stride=640, out_stride=640), INVALID),
    (dict(head_dim=80), UNSUPPORTED), (dict(q_stride=504), INVALID),
    (dict(out_stride=516), UNSUPPORTED), (dict(out_stride=520), INVALID),
    (dict(max_pages=0), INVALID), (dict(max_pages=2 ** 25), UNSUPPORTED),
    (dict(num_pages=0), INVALID), (dict(num_pages=2 ** 26), UNSUPPORTED),
    (dict(page=48), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=3e38), INVALID), (dict(scale=INF), INVALID), (dict(scale=NAN), INVALID), (dict(causal=2), INVALID),
    (dict(q=None), INVALID), (dict(q_offsets=None), INVALID), (dict(q_offsets=P + 4), INVALID),
    (dict(lengths=None), INVALID), (dict(pages=None), INVALID), (dict(cache=None), INVALID),
    (dict(out=None), INVALID), (dict(max_pages=300, workspace=None), WORKSPACE),
    (dict(max_pages=300, workspace_bytes=1024), WORKSPACE),
    (dict(max_pages=300, workspace=P + 16), INVALID),
    (dict(n=0, q=None, q_offsets=P, out=None, workspace=None), OK),
    (dict(n=0, batch=0, q_offsets=None, lengths=None, pages=None, workspace=None), OK)])
def test_cache_attention_refuses(kw, status):
    a = dict(ATTENTION)
    a.update(kw)
    assert _status(lk.lookme_cache_attention, *a.values(), 0) == status


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_workspace_has_one_bound(dtype, d):
    """the constant serves every call; small and large ones need none"""
    most = 0
    for n, batch in ((1, 1), (64, 64), (2048, 2048), (7, 1), (35, 7), (600, 2), (10 ** 5, 4),
                     (2 ** 16, 2 ** 16), (2 ** 21, 2 ** 16)):
        for hq, hkv in ((1, 1), (8, 1), (32, 8), (64, 64)):
            for pages in (1, 4, 2 ** 14):
                b = lk.lookme_cache_attention_workspace(dtype, n, batch, hq, hkv, d, pages, 32)
                assert 0 <= b <= lk.LOOKME_ATTENTION_WORKSPACE
                most = max(most, b)
    for n in (2 ** 22, 2 ** 25, 2 ** 27):
        for page in (32, 1024):
            b = lk.lookme_cache_attention_workspace(dtype, n, 2 ** 22, 1, 1, d, 2 ** 20, page)
            assert 0 <= b <= lk.LOOKME_ATTENTION_WORKSPACE
    assert most > 0
    assert lk.lookme_cache_attention_workspace(dtype, 0, 0, 8, 1, d, 4, 32) == 0


def test_workspace_size_refuses():
    assert _status(lk.lookme_cache_attention_workspace, 2, 4, 4, 8, 1, 128, 4, 32) == INVALID
    assert _status(lk.lookme_cache_attention_workspace, BF, 4, 4, 8, 3, 128, 4, 32) == INVALID
    assert lk.load().lookme_cache_attention_workspace(BF, 4, 4, 8, 1, 128, 4, 32, None) == INVALID


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


I32, U8, F = torch.int32, torch.uint8, torch.float32
CACHE_T = dict(cache=_t(2, 2, 1, 34 * 64, dtype=U8))


def _attend(**kw):
    a = dict(q=_t(3, 4, 64), cache=_t(2, 2, 1, 34 * 64, dtype=U8), pages=_t(3, 2, dtype=I32),
             lengths=_t(3, dtype=I32), out=_t(3, 4, 64))
    a.update(kw)
    return lk.cache_attention(**a)


@pytest.mark.parametrize("call", [
    lambda: lk.head_norm_rotary(_t(3, 4, 64), _t(3, 4, 64)),                     # on the CPU
    lambda: lk.head_norm_rotary(_t(3, 64), _t(3, 64)),
    lambda: lk.head_norm_rotary(_t(3, 4, 64, dtype=torch.float16), _t(3, 4, 64)),
    lambda: lk.head_norm_rotary(_t(3, 4, 64), _t(3, 4, 32)),
    lambda: lk.head_norm_rotary(_t(3, 8, 64)[:, ::2], _t(3, 4, 64)),             # heads apart
    lambda: lk.head_norm_rotary(_t(3, 4, 128)[..., ::2], _t(3, 4, 64)),
    lambda: lk.head_norm_rotary(_t(1, 4, 64).expand(3, 4, 64), _t(3, 4, 64)),    # rows overlap
    lambda: lk.head_norm_rotary(_t(3, 4, 64), _t(3, 4, 64), k=_t(3, 2, 64)),
    lambda: lk.head_norm_rotary(_t(3, 4, 64), _t(3, 4, 64), k_weight=_t(64)),
    lambda: lk.head_norm_rotary(_t(3, 4, 64), _t(3, 4, 64), k=_t(2, 2, 64), k_out=_t(2, 2, 64)),
    lambda: lk.head_norm_rotary(_t(3, 4, 64), _t(3, 4, 64), q_weight=_t(32)),
    lambda: lk.head_norm_rotary(_t(3, 4, 64), _t(3, 4, 64), freq=_t(32, dtype=F)),
    lambda: lk.head_norm_rotary(_t(3, 4, 64), _t(3, 4, 64), pos=_t(3, dtype=I32)),
    lambda: lk.head_norm_rotary(_t(3, 4, 64), _t(3, 4, 64), freq=_t(32, dtype=F),
                                pos=_t(4, dtype=I32)),
    lambda: lk.head_norm_rotary(_t(3, 4, 64), _t(3, 4, 64), freq=_t(32, dtype=F),
                                pos=_t(3, dtype=torch.int64)),
    lambda: lk.head_norm_rotary(_t(3, 4, 64), _t(3, 4, 64), freq=_t(32, dtype=F),
                                pos=_t(3, 3, dtype=I32)),                        # no axis
    lambda: lk.head_norm_rotary(_t(3, 4, 64), _t(3, 4, 64), freq=_t(32, dtype=F),
                                pos=_t(3, 3, dtype=I32), axis=_t(16, dtype=I32)),
    lambda: lk.cache_write(_t(3, 2, 64), _t(3, 2, 64), _t(3, dtype=I32), **CACHE_T),
    lambda: lk.cache_write(_t(3, 1, 64), _t(3, 1, 64), _t(3, dtype=I32), **CACHE_T),
    lambda: lk.cache_write(_t(3, 2, 64), _t(2, 2, 64), _t(3, dtype=I32), **CACHE_T),
    lambda: lk.cache_write(_t(3, 2, 64), _t(3, 2, 64), _t(2, dtype=I32), **CACHE_T),
    lambda: lk.cache_write(_t(3, 2, 64), _t(3, 2, 64), _t(3, dtype=I32),
                           _t(2, 2, 1, 33 * 64, dtype=U8)),
    lambda: lk.cache_write(_t(3, 2, 64), _t(3, 2, 64), _t(3, dtype=I32),
                           _t(2, 2, 34 * 64, dtype=U8)),
    lambda: lk.cache_read(_t(3, dtype=I32), **CACHE_T),
    lambda: lk.cache_read(_t(3, dtype=I32), k_out=_t(2, 2, 64), **CACHE_T),
    lambda: lk.cache_read(_t(3, dtype=I32), k_out=_t(3, 2, 64), v_out=_t(3, 2, 64, dtype=F),
                          **CACHE_T),
    lambda: _attend(), lambda: _attend(q=_t(3, 4, 128)), lambda: _attend(out=_t(3, 2, 64)),
    lambda: _attend(lengths=_t(2, dtype=I32)), lambda: _attend(pages=_t(6, dtype=I32)),
    lambda: _attend(pages=_t(3, 4, dtype=I32)[:, ::2]),
    lambda: _attend(q_offsets=_t(3, dtype=I32)), lambda: _attend(workspace=_t(64)),
])
def test_bindings_refuse(call):
    assert _status(call) == INVALID


BIG = 2 ** 32
RAW = {"lookme_head_norm_rotary": list(ROTARY.values()),
       "lookme_cache_write": [BF, 5, 2, 128, P, 256, P, 256, P, 8, 32, P],
       "lookme_cache_read": [BF, 5, 2, 128, P, 8, 32, P, P, 256, P, 256],
       "lookme_cache_attention": list(ATTENTION.values()),
       "lookme_cache_attention_workspace": [BF, 6, 2, 4, 2, 128, 3, 64]}
SIZES = [("lookme_head_norm_rotary", i) for i in (0, 2, 3, 8, 13, 17, 18, 19)]
SIZES += [("lookme_cache_write", i) for i in (0, 2, 3, 10)]
SIZES += [("lookme_cache_read", i) for i in (0, 2, 3, 6)]
SIZES += [("lookme_cache_attention", i) for i in (0, 2, 3, 4, 5, 11, 13, 16)]
SIZES += [("lookme_cache_attention_workspace", i) for i in (0, 2, 3, 4, 5, 6, 7)]


@pytest.mark.parametrize("name,at", SIZES)
def test_sizes_past_32_bits_are_refused(monkeypatch, name, at):
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or OK

    monkeypatch.setattr(lk, "_lib", Library())
    args, more = list(RAW[name]), {} if name.endswith("workspace") else {"stream": 0}
    getattr(lk, name)(*args, **more)
    for v in (BIG + args[at], args[at] - BIG):
        args[at] = v
        with pytest.raises(lk.LookmeError) as e:
            getattr(lk, name)(*args, **more)
        assert e.value.status == INVALID
    assert calls == [name]


# ---- the plain forms ---------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128, 256])
def test_the_tile_has_a_place_for_every_byte(d):
    """places() is a one-to-one map onto the 34 d bytes"""
    at = torch.cat([torch.cat(A.places(t, d)) for t in range(32)])
    assert torch.equal(at.sort().values, torch.arange(34 * d))


def test_quantize_rounds_to_the_nearest_even_code():
    x = torch.zeros(2, 64)
    x[0, :12] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -2.5, 5.01, 0.26])
    x[0, 32] = 7.0
    x[1, 0], x[1, 32] = 7.01, 3.5
    code, byte = A.quantize(x)
    assert byte.tolist() == [[127, 127], [128, 126]]
    assert code[0, :12].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 12, 7, 1]
    assert code[0, 32] == 7 and code[1, 0] == 5 + 1 and code[1, 32] == 7
    assert A.value(code, byte)[0, :8].tolist() == [6, 0, 1, 1, 2, 2, 4, 4]
    x[0, 5], x[1, 40] = NAN, INF
    code, byte = A.quantize(x)
    assert byte.tolist() == [[255, 127], [128, 255]] and not code[0, :32].any()
    assert A.value(code, byte)[0, :32].isnan().all()
    code, byte = A.quantize(torch.full((32,), 3e38))
    assert byte == 252 and (code == 7).all()
    code, byte = A.quantize(torch.full((32,), 1e-38))
    assert byte == 27 and (code == 0).all()


def test_the_cache_gives_back_what_it_holds():
    g = torch.Generator().manual_seed(0)
    for d in (64, 128, 256):
        k, v = torch.randn((40, 2, d), generator=g), torch.randn((40, 2, d), generator=g)
        slots = torch.randperm(128, generator=g)[:40]
        cache = A.write(torch.zeros((2, 2, 2, 34 * d), dtype=torch.uint8), slots, k, v)
        rk, rv = A.read(cache, slots)
        for x, r in ((k, rk), (v, rv)):
            assert torch.equal(r, A.value(*A.quantize(x)))
            top = x.abs().unflatten(-1, (-1, 32)).amax(-1, keepdim=True).double()
            assert ((r - x).abs().unflatten(-1, (-1, 32)) <= top / 3.5).all()


def test_plain_forms_agree_with_torch():
    g = torch.Generator().manual_seed(1)
    q = torch.randn((5, 4, 64), generator=g)
    k, v = torch.randn((9, 2, 64), generator=g), torch.randn((9, 2, 64), generator=g)
    out, bound = A.attention(q, k.double(), v.double(), 0.125, True)
    mask = torch.ones(5, 9).tril(4).bool()
    t = lambda x: x.transpose(0, 1)[None].double()  # noqa: E731
    want = torch.nn.functional.scaled_dot_product_attention(
        t(q), t(k).repeat_interleave(2, 1), t(v).repeat_interleave(2, 1), attn_mask=mask,
        scale=0.125)[0].transpose(0, 1)
    assert (out - want).abs().max() < 1e-12 and (bound > 0).all()
    out, _ = A.attention(q, k[:2].double(), v[:2].double(), 0.125, True)
    assert not out[:3].any() and torch.allclose(out[3, 0], v[0, 0].double())
    # a rotation by a position keeps lengths, and one by nothing changes nothing
    pos, freq = torch.tensor([0, 3, 7, -2, 10 ** 6], dtype=torch.int32), torch.rand(16, generator=g)
    for inter in (False, True):
        y, _ = A.rotary(q, pos=pos, freq=freq, interleaved=inter)
        assert torch.allclose(y.norm(dim=-1), q.double().norm(dim=-1))
        assert torch.equal(y[0], q[0].double()) and torch.equal(y[..., 32:], q[..., 32:].double())
        z = torch.view_as_complex(torch.stack(
            [q[1, 0, 0:32:2], q[1, 0, 1:32:2]] if inter else [q[1, 0, :16], q[1, 0, 16:32]], -1
        ).double()) * torch.exp(1j * 3 * freq.double())
        got = (y[1, 0, 0:32:2], y[1, 0, 1:32:2]) if inter else (y[1, 0, :16], y[1, 0, 16:32])
        assert torch.allclose(got[0], z.real) and torch.allclose(got[1], z.imag)
    y, e = A.rotary(q, weight=torch.ones(64), eps=0.0)
    assert ((torch.nn.functional.rms_norm(q, (64,), eps=0.0) - y).abs() <= e).all()
    assert math.isclose(float(y[0, 0].norm()), 8.0)
