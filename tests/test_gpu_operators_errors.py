"""GPU tests of what the operators around a LookME layer report: the status of their
own launches."""

import ctypes

import pytest
import torch

from tests.test_gpu_operators_chain import Decode, Experts, lk  # noqa: F401

pytestmark = pytest.mark.gpu


def test_an_error_that_others_left_is_not_reported(lk):  # noqa: F811
    """a failed call of the program's own (a device that does not exist is made current)
    leaves the thread's last error; the operators run, succeed and leave it alone"""
    hip = ctypes.CDLL(lk.LIB_PATH)   # the runtime that the library is linked to
    s, d = Experts(), Decode(3)
    s.route(lk)
    torch.cuda.synchronize()
    assert hip.hipSetDevice(ctypes.c_int(9999)) != 0
    assert hip.hipPeekAtLastError() != 0
    try:
        s.run(lk)
        d.run(lk)
        assert hip.hipPeekAtLastError() != 0
    finally:
        hip.hipGetLastError()
    torch.cuda.synchronize()
    s.check()
    d.check()
