"""Refusals of the context-free operators that need no device, beyond tests/test_operators_cpu.py."""
import ctypes as C

import pytest

import paper_2403_09054_b200 as kf
from tests.test_operators_cpu import FAR, _step


@pytest.mark.parametrize("value", [-1, 2])
def test_packed_step_self_test_argument(value):
    a = _step(debug_fail_first_wait=value)
    assert kf.LIB.kf_packed_scratch_bytes(C.byref(a)) == 0
    assert kf.LIB.kf_decode_step_packed(C.byref(a), *FAR[:8], None, None, None, FAR[11], 1 << 30, None) == kf.KF_EINVAL
