"""Refusals of the operators around attention that are made before anything
reaches a device, asked of the library through its C entry points."""
import ctypes as C

import pytest

from paper_2606_09514_amd import lib as blib

P = 0x10000                                                    # never followed


class Norm(C.Structure):
    _fields_ = [("n_rows", C.c_int32), ("width", C.c_int32), ("hidden_dtype", C.c_int32), ("dtype", C.c_int32),
                ("h", C.c_void_p), ("delta", C.c_void_p), ("weight", C.c_void_p), ("h_out", C.c_void_p), ("y", C.c_void_p),
                ("y_mx8", C.c_void_p), ("h_stride", C.c_int64), ("delta_stride", C.c_int64), ("h_out_stride", C.c_int64),
                ("y_stride", C.c_int64), ("pos", C.c_void_p), ("rms_eps", C.c_float)]


@pytest.mark.parametrize("hidden", [blib.F32, blib.BF16])
def test_norm_refuses_a_sum_in_place_with_rows_elsewhere(hidden):
    """h_out = h with another stride: rows would be written over rows that other
    workgroups have yet to read."""
    call = lambda **k: blib.lib().buddy_add_rmsnorm(
        C.byref(Norm(**{**dict(n_rows=3, width=48, hidden_dtype=hidden, dtype=blib.BF16, h=P, delta=P, weight=P, h_out=P, y=P, h_stride=48,
                               delta_stride=48, h_out_stride=48, y_stride=48, rms_eps=1e-6), **k})), None)
    assert call(h_out_stride=64) == blib.EINVAL
    assert call(h_stride=4096) == blib.EINVAL
    assert call(n_rows=0, h_out_stride=64) == blib.OK
