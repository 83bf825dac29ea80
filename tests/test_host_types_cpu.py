"""The host entry points and element types that only the network operators take (no GPU)."""
import ctypes

import numpy as np
import pytest

INVALID, F16, BF16 = 1, 2, 3


@pytest.mark.parametrize("dtype", [F16, BF16, 7, -1])
@pytest.mark.parametrize("entry", ["ndvm_value_and_grad_host", "ndvm_value_and_grad_host_async"])
def test_host_replay_refuses_other_types_before_it_reads(ndvm, entry, dtype):
    """A 16-bit buffer holds a quarter of what a copy of doubles would read."""
    lib, tape = ndvm.load(), ndvm.trace_build("(model (params a b) (* a b))")
    params, out, grad = np.ones(8, np.float16), np.ones(4, np.float16), np.ones(8, np.float16)
    ptr = [ctypes.c_void_p(a.ctypes.data) for a in (params, out, grad)]
    assert getattr(lib, entry)(tape.handle, dtype, 4, ptr[0], None, 0, ptr[1], ptr[2], None) == INVALID
    assert b"dtype" in lib.ndvm_last_error()
