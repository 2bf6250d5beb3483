"""Refusals of the operators around attention that are made before anything
reaches a device, asked of the library through its C entry points."""
import ctypes as C
import os

import pytest

from paper_2606_09514_amd import lib as blib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
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


def test_calls_take_as_many_rows_as_the_header_says():
    """Up to 2^24 rows, of projections, adapters and plans 2^20.  The largest are
    taken (asked for their workspace, or given nothing to point at), one more is
    refused."""
    L, big, most = blib.lib(), 1 << 20, 1 << 24
    eight = lambda rows, width=64: blib.MX8Struct(P, P, width, 16, rows, width)
    space = lambda x, w: L.buddy_mx8_linear_workspace(C.byref(x), C.byref(w))
    assert space(eight(big), eight(8)) > 0 and space(eight(8), eight(big)) > 0
    assert space(eight(big + 1), eight(8)) == 0 and space(eight(8), eight(big + 1)) == 0
    linear = lambda x, w: L.buddy_mx8_linear(C.byref(x), C.byref(w), blib.BF16, None, C.c_int64(8), None, C.c_size_t(0), None)
    assert linear(eight(big), eight(8)) == blib.EINVAL and linear(eight(big + 1), eight(8)) == blib.ECAPACITY
    assert linear(eight(8), eight(big)) == blib.EINVAL and linear(eight(8), eight(big + 1)) == blib.ECAPACITY
    l = blib.LoraStruct(P, P, P, blib.BF16, 3, 16, 1 << 20, 1 << 20)
    assert L.buddy_lora_workspace(C.byref(l), big) > 0 and L.buddy_lora_workspace(C.byref(l), big + 1) == 0
    assert L.buddy_lora_plan_size(big, 4096) > 0 and L.buddy_lora_plan_size(big + 1, 4096) == 0
    assert L.buddy_lora_plan(None, big, 3, None, None) == blib.EINVAL and L.buddy_lora_plan(None, big + 1, 3, None, None) == blib.ECAPACITY
    norm = lambda n: L.buddy_add_rmsnorm(C.byref(Norm(n_rows=n, width=64, hidden_dtype=blib.F32, dtype=blib.BF16, y=P)), None)
    assert norm(most) == blib.EINVAL and norm(most + 1) == blib.ECAPACITY
    quantise = lambda n: L.buddy_mx8_quantize(C.byref(eight(n)), blib.BF16, None, C.c_int64(64), None, C.c_int64(0), None, None)
    assert quantise(most) == blib.EINVAL and quantise(most + 1) == blib.ECAPACITY
    read = lambda n: L.buddy_mx8_read(C.byref(eight(n)), blib.BF16, None, C.c_int64(64), None)
    assert read(most) == blib.EINVAL and read(most + 1) == blib.ECAPACITY


def test_the_header_says_these_limits():
    text = " ".join(open(os.path.join(ROOT, "include", "buddy.h")).read().replace("*", " ").split())
    assert "A call takes up to 2^24 rows, of projections (rows of weights, too), adapters and their plans 2^20 (BUDDY_ECAPACITY)" in text
