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
    assert calls == [("lookme_group_rows", (8, 1234)), ("lookme_group_rows", (8, 77))]
