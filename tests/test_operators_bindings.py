"""What the torch bindings of the operators around a LookME layer pass on, without
a GPU: streams of other devices and sizes past 32 bits are refused before the
library is called."""

import types

import pytest
import torch

from paper_2607_16305_amd import lookme as lk


@pytest.fixture
def calls(monkeypatch):
    """the library's calls, recorded instead of made; device 0 is current"""
    got = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: got.append((name, a)) or lk.LOOKME_OK

    monkeypatch.setattr(lk, "_lib", Library())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0)
    return got


def _stream(device):
    return types.SimpleNamespace(device_index=device, cuda_stream=1234)


def test_a_stream_of_another_device_is_refused(calls):
    with pytest.raises(lk.LookmeError) as e:
        lk._call("lookme_group_rows", 0, _stream(1), 8, 0, None, None, 0)
    assert e.value.status == lk.LOOKME_ERR_INVALID and "stream" in str(e.value)
    assert not calls


def test_a_stream_of_the_tensors_device_and_an_address_are_passed_on(calls):
    lk._call("lookme_group_rows", 0, _stream(0), 8)
    lk._call("lookme_group_rows", 0, 77, 8)
    lk._call("lookme_group_rows", 0, types.SimpleNamespace(cuda_stream=5), 8)   # says no device
    assert [c[1] for c in calls] == [(8, 1234), (8, 77), (8, 5)]


BIG = 2 ** 32           # cut to 32 bits, BIG + 64 is 64
RAW = {
    "lookme_residual_norm": (lk.LOOKME_BF16, 4, 64, 16, 1, 16, None, None, 1e-6, 16, None, None,
                             None),
    "lookme_group_rows": (8, 16, 16, 16, 16),
    "lookme_grouped_product": (lk.LOOKME_BF16, 8, 16, 64, 32, 16, 16, 16, 1, 16, 16, None, 16, 0),
    "lookme_grouped_product_quant": (8, 16, 64, 32, 16, 16, 16, 16, 1, 16, 16, 16, None, None, 16,
                                     0),
    "lookme_quant_product": (lk.LOOKME_BF16, 4, 256, 32, 64, 16, 16, 16, None, None, 16),
    "lookme_quant_swiglu": (lk.LOOKME_BF16, 4, 256, 32, 64, 16, 16, 16, None, 16, 16, None, 16),
}
SIZES = [("lookme_residual_norm", 0), ("lookme_residual_norm", 2), ("lookme_residual_norm", 4),
         ("lookme_group_rows", 0)]
SIZES += [("lookme_grouped_product", i) for i in (0, 1, 3, 4, 8, 13)]
SIZES += [("lookme_grouped_product_quant", i) for i in (0, 2, 3, 8, 15)]
SIZES += [(f, i) for f in ("lookme_quant_product", "lookme_quant_swiglu") for i in (0, 2, 3, 4)]


@pytest.mark.parametrize("name,at", SIZES)
def test_sizes_past_32_bits_are_refused(calls, name, at):
    args = list(RAW[name])
    getattr(lk, name)(*args, stream=0)
    assert [c[0] for c in calls] == [name]
    for v in (BIG + args[at], args[at] - BIG):
        args[at] = v
        with pytest.raises(lk.LookmeError) as e:
            getattr(lk, name)(*args, stream=0)
        assert e.value.status == lk.LOOKME_ERR_INVALID
    assert len(calls) == 1


class Shape:
    """what a binding asks of a tensor, of any size"""

    def __init__(self, *shape, dtype=torch.bfloat16):
        self.shape, self.dtype = torch.Size(shape), dtype

    def get_device(self):
        return 0

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 16


I32, U8, N = torch.int32, torch.uint8, 64


@pytest.mark.parametrize("call", [
    lambda b: lk.residual_norm(Shape(4, b + N), out=Shape(4, b + N)),
    lambda b: lk.residual_norm(Shape(4, N), add=Shape(4, b + 2, N), out=Shape(4, N)),
    lambda b: lk.group_rows(Shape(8, dtype=I32), b + 4, Shape(8, dtype=I32),
                            Shape(b + 5, dtype=I32)),
    lambda b: lk.grouped_product(Shape(8, b + N), Shape(2, 32, b + N), Shape(3, dtype=I32),
                                 Shape(8, 32)),
    lambda b: lk.grouped_product(Shape(8, N), Shape(2, b + 32, N), Shape(3, dtype=I32),
                                 Shape(8, b + 32)),
    lambda b: lk.grouped_product(Shape(8, N), Shape(b + 2, 32, N), Shape(b + 3, dtype=I32),
                                 Shape(8, 32)),
    lambda b: lk.grouped_product(Shape(8, N), Shape(2, 32, N), Shape(3, dtype=I32), Shape(8, 32),
                                 rows=Shape(8, dtype=I32), picks=b + 2),
    lambda b: lk.quant_product(Shape(2, b + N), Shape(8, b // 2 + N // 2, dtype=U8),
                               Shape(8, b // 32 + 2), Shape(2, 8)),
    lambda b: lk.quant_product(Shape(2, N), Shape(b + 8, N // 2, dtype=U8), Shape(b + 8, 2),
                               Shape(2, b + 8)),
    lambda b: lk.quant_swiglu(Shape(2, N), *[Shape(b + 8, N // 2, dtype=U8), Shape(b + 8, 2)] * 2,
                              Shape(2, b + 8)),
])
def test_tensors_of_sizes_past_32_bits_are_refused(calls, call):
    call(0)
    assert len(calls) == 1
    with pytest.raises(lk.LookmeError):
        call(BIG)
    assert len(calls) == 1
