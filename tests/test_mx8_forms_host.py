"""Which form a projection of 8-bit rows takes, asked of the library without a
device: the shapes of the device tests reach every kernel."""
import ctypes as C

import pytest
import torch

from paper_2606_09514_amd import lib as blib
from test_mx8_forms_gpu import BATCH, BATCHES, FAR, FORMS, STREAM, TILE, TILES

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Rows:
    """Sizes and strides of 8-bit rows; no memory behind them."""

    def __init__(self, rows, width, stride=0, scale_stride=0):
        self.struct = blib.MX8Struct(None, None, stride or width, scale_stride or (width + 511) // 512 * 16, rows, width)


def form_of(x, w, dtype):
    f = blib.mx8_linear_form(x, w, dtype)
    return f.form, f.row_tiles, f.weight_tiles, f.parts, f.splits


def test_shapes_take_the_forms_that_they_are_listed_for():
    for dtype, rows, n, k, form in FORMS:
        assert form_of(Rows(rows, k), Rows(n, k), DT[dtype]) == form, (dtype, rows, n, k)


def test_the_shapes_reach_every_kernel():
    """Each kernel that the library has, with sums of splits of k and without
    where a split can be, and six to eight wavefronts of one part."""
    have = {(f[0], f[1], f[3], dtype) for dtype, *_, f in FORMS}
    batch = {(BATCH, tiles, parts, d) for d in DT for tiles, most in ((1, 8), (2, 4), (4, 4), (6, 2), (8, 2)) for parts in (1, 2, 4, 8) if parts <= most}
    assert have == batch | {(STREAM, 1, 8, d) for d in DT} | {(TILE, 16, 1, "bf16")}
    split = {(f[0], f[1], dtype) for dtype, *_, f in FORMS if f[4] > 1}
    assert split == {(BATCH, t, d) for d in DT for t in (1, 2, 4, 6, 8)} | {(TILE, 16, "bf16")}
    assert {f[2] for *_, f in FORMS if f[0] == BATCH and f[3] == 1} == {6, 7, 8}
    for dtype, rows, n, k in [("bf16", *t[:3]) for t in TILES] + BATCHES:
        assert form_of(Rows(rows, k), Rows(n, k), DT[dtype])[0] == (TILE if (rows, n, k) in [t[:3] for t in TILES] else BATCH)
    for rows, n, k, splits in TILES:
        assert form_of(Rows(rows, k), Rows(n, k), torch.bfloat16)[4] == splits
    assert len({form_of(Rows(*c[1::2]), Rows(*c[2:]), DT[c[0]])[1] for c in BATCHES}) >= 3


def test_rows_far_apart_and_few_rows():
    x, w = Rows(600, 4096), Rows(28672, 4096)
    assert form_of(x, w, torch.bfloat16)[0] == TILE
    for far in (dict(stride=FAR), dict(scale_stride=FAR)):
        assert form_of(Rows(600, 4096, **far), w, torch.bfloat16) == (STREAM, 2, 1, 4, 1)
        assert form_of(x, Rows(28672, 4096, **far), torch.float32) == (STREAM, 2, 1, 4, 1)
        assert form_of(Rows(16, 4096, **far), w, torch.bfloat16) == (STREAM, 1, 1, 8, 1)
    assert form_of(Rows(600, 4096, stride=2 ** 23 - 16), w, torch.bfloat16)[0] == TILE
    assert form_of(Rows(600, 4096), w, torch.float32)[0] == BATCH            # tiles are of bf16 outputs


def test_form_refuses_what_the_call_refuses():
    ask = lambda x, w, t, f: blib.lib().buddy_mx8_linear_form(C.byref(x.struct) if x else None, C.byref(w.struct) if w else None, t, f)
    f = blib.MX8Form(9, 9, 9, 9, 9)
    out = C.byref(f)
    assert ask(None, Rows(1, 16), 0, out) == ask(Rows(1, 16), None, 0, out) == blib.EINVAL
    assert ask(Rows(1, 16), Rows(1, 32), 0, out) == ask(Rows(1, 16), Rows(0, 16), 0, out) == blib.EINVAL
    assert ask(Rows(1, 24), Rows(1, 24), 0, out) == blib.ESHAPE
    assert ask(Rows(2 ** 20 + 1, 16), Rows(1, 16), 0, out) == blib.ECAPACITY
    assert ask(Rows(1, 16), Rows(1, 16), 2, out) == ask(Rows(1, 16), Rows(1, 16), 0, None) == blib.EINVAL
    assert f.form == 9
    assert ask(Rows(0, 16), Rows(1, 16), 0, out) == blib.OK
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        blib.mx8_linear_form(Rows(1, 16), Rows(1, 16), torch.float16)
    with pytest.raises(blib.BuddyError):
        blib.mx8_linear_form(Rows(1, 24), Rows(1, 24), torch.float32)
