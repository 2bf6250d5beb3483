"""Every form of the projection of 8-bit rows on the device: which kernel a shape
takes is asked of the library, so that a planner measured anew cannot leave one
without a test.

Tolerances as for the operators around attention: fp32 outputs (K + 16) u sum |p|,
bf16 outputs 2^-10 sum over eights of max |p| + (K / 8 + 64) u sum |p|, then the
output's rounding.  A split of k adds at most 8 additions to the K / 8 or K that
are counted, whose order is free.  On all outputs the maxima of eights are bounded
by sum |p|, on a sample of rows they are taken."""
import math

import pytest
import torch

from paper_2606_09514_amd import lib as blib
from test_serving_gpu import DT, E4M3, ROUND, U, gen, mx8_of, run_linear

pytestmark = pytest.mark.gpu

STREAM, BATCH, TILE = 0, 1, 2
# type, rows, weight rows, k: form, tiles of 16 rows and of 16 weight rows, parts of k, splits
FORMS = [
    ("bf16", 1, 1, 16, (STREAM, 1, 1, 8, 1)), ("f32", 1, 1, 16, (STREAM, 1, 1, 8, 1)),
    ("bf16", 70, 5486, 1088, (BATCH, 4, 4, 2, 1)), ("f32", 70, 5486, 1088, (BATCH, 1, 7, 1, 1)),
    ("f32", 15, 17166, 3568, (BATCH, 1, 6, 1, 1)), ("bf16", 2, 16421, 2544, (BATCH, 1, 6, 1, 1)),
    ("f32", 807, 626, 1216, (BATCH, 1, 8, 1, 1)), ("bf16", 1, 28681, 1312, (BATCH, 1, 8, 1, 1)),
    ("bf16", 1, 24621, 1232, (BATCH, 1, 7, 1, 1)),
    ("bf16", 19, 1, 1808, (BATCH, 1, 4, 2, 1)), ("f32", 19, 1, 1808, (BATCH, 1, 4, 2, 1)),
    ("bf16", 17, 2, 3600, (BATCH, 1, 2, 4, 1)), ("f32", 17, 2, 3600, (BATCH, 1, 2, 4, 1)),
    ("bf16", 17, 1, 7200, (BATCH, 1, 1, 8, 1)), ("f32", 17, 1, 7200, (BATCH, 1, 1, 8, 1)),
    ("bf16", 17, 2, 14368, (BATCH, 1, 1, 8, 2)), ("f32", 17, 2, 14368, (BATCH, 1, 1, 8, 2)),
    ("bf16", 19, 4, 65536, (BATCH, 1, 1, 8, 8)), ("f32", 19, 4, 65536, (BATCH, 1, 1, 8, 8)),
    ("bf16", 19, 16413, 1424, (BATCH, 2, 6, 1, 1)), ("f32", 697, 725, 1056, (BATCH, 2, 6, 1, 1)),
    ("bf16", 133, 5697, 1120, (BATCH, 2, 7, 1, 1)), ("f32", 897, 794, 1088, (BATCH, 2, 7, 1, 1)),
    ("bf16", 527, 1845, 1184, (BATCH, 2, 8, 1, 1)), ("f32", 954, 914, 1056, (BATCH, 2, 8, 1, 1)),
    ("bf16", 458, 537, 1856, (BATCH, 2, 4, 2, 1)), ("f32", 458, 537, 1856, (BATCH, 2, 4, 2, 1)),
    ("bf16", 354, 354, 3680, (BATCH, 2, 2, 4, 1)), ("f32", 354, 354, 3680, (BATCH, 2, 2, 4, 1)),
    ("bf16", 1052, 58, 10288, (BATCH, 2, 2, 4, 2)), ("f32", 113, 539, 10256, (BATCH, 2, 2, 4, 2)),
    ("bf16", 38, 16474, 960, (BATCH, 4, 6, 1, 1)), ("f32", 961, 1493, 1104, (BATCH, 4, 6, 1, 1)),
    ("bf16", 306, 5442, 912, (BATCH, 4, 7, 1, 1)), ("f32", 1353, 1134, 1088, (BATCH, 4, 7, 1, 1)),
    ("bf16", 1412, 1369, 960, (BATCH, 4, 8, 1, 1)), ("f32", 1251, 1345, 1136, (BATCH, 4, 8, 1, 1)),
    ("bf16", 741, 673, 1824, (BATCH, 4, 4, 2, 1)), ("f32", 741, 673, 1824, (BATCH, 4, 4, 2, 1)),
    ("bf16", 633, 398, 3728, (BATCH, 4, 2, 4, 1)), ("f32", 633, 398, 3728, (BATCH, 4, 2, 4, 1)),
    ("bf16", 38, 1448, 9216, (BATCH, 4, 2, 4, 4)), ("f32", 692, 186, 10336, (BATCH, 4, 2, 4, 2)),
    ("bf16", 1131, 1891, 928, (BATCH, 6, 6, 1, 1)), ("f32", 1131, 1891, 928, (BATCH, 6, 6, 1, 1)),
    ("bf16", 1169, 1887, 912, (BATCH, 6, 7, 1, 1)), ("f32", 1233, 2201, 976, (BATCH, 6, 8, 1, 1)),
    ("bf16", 1078, 966, 1808, (BATCH, 6, 4, 2, 1)), ("f32", 1078, 966, 1808, (BATCH, 6, 4, 2, 1)),
    ("bf16", 76, 5792, 9216, (BATCH, 6, 4, 2, 2)), ("f32", 76, 5792, 9216, (BATCH, 6, 4, 2, 2)),
    ("bf16", 877, 3423, 912, (BATCH, 8, 6, 1, 1)), ("f32", 877, 3423, 912, (BATCH, 8, 6, 1, 1)),
    ("bf16", 1165, 2471, 1040, (BATCH, 8, 7, 1, 1)), ("f32", 1243, 2823, 944, (BATCH, 8, 8, 1, 1)),
    ("bf16", 1150, 1353, 1904, (BATCH, 8, 4, 2, 1)), ("f32", 1150, 1353, 1904, (BATCH, 8, 4, 2, 1)),
    ("bf16", 107, 1217, 13824, (BATCH, 8, 4, 2, 8)), ("f32", 107, 1217, 13824, (BATCH, 8, 4, 2, 8)),
    ("bf16", 1401, 3275, 512, (TILE, 16, 16, 1, 1)), ("bf16", 600, 28672, 4096, (TILE, 16, 16, 1, 1)),
    ("bf16", 304, 13777, 5120, (TILE, 16, 16, 1, 2)), ("bf16", 430, 3444, 13824, (TILE, 16, 16, 1, 8))]
TILES = [(1401, 3275, 640, 1), (304, 13777, 5120, 2), (198, 2706, 14464, 8)]
BATCHES = [("bf16", 38, 16474, 960), ("f32", 1131, 1891, 928), ("bf16", 107, 1217, 13824), ("f32", 76, 5792, 9216)]
FAR = 2 ** 23 + 4096


def form_of(x, w, dtype):
    f = blib.mx8_linear_form(x, w, dtype)
    return f.form, f.row_tiles, f.weight_tiles, f.parts, f.splits


def rows_of(rows, k, g):
    x = torch.randn((rows, k), generator=g).cuda()
    spread = torch.randint(-2, 3, (rows, (k + 31) // 32), generator=g).cuda().float()
    return mx8_of(x * torch.exp2(spread).repeat_interleave(32, 1)[:, :k])


def values(m):
    """8-bit rows as 64-bit values, on the device."""
    table = torch.cat((E4M3, torch.tensor([math.nan]), -E4M3, torch.tensor([math.nan]))).cuda()
    s = torch.exp2(m._keep[1].double() - 127)
    s[m._keep[1] == 255] = math.nan
    x = table[m._keep[0].int()]
    return x.mul_(s.repeat_interleave(32, 1)[:, :m.shape[1]])


def check_linear(x, w, out):
    """All outputs, and a sample of rows with the maxima of eights."""
    dtype, k, n = out.dtype, x.shape[1], w.shape[0]
    xv, wv = values(x), values(w)
    want, total = xv @ wv.T.contiguous(), xv.abs() @ wv.T.abs().contiguous()
    assert not want.isnan().any()
    fine = ROUND[dtype] * want.abs() + ((k + 16) if dtype is torch.float32 else (k / 8 + 64)) * U * total
    err = (out.double() - want).abs()
    if dtype is torch.float32:
        assert (err <= fine).all(), float((err - fine).max())
        return
    assert (err <= fine + 2.0 ** -10 * total).all(), float((err - fine - 2.0 ** -10 * total).max())
    rows = sorted({r for r in (0, 1, 15, 16, 63, 64, 127, 128, 255, 256, x.shape[0] // 2, x.shape[0] - 2, x.shape[0] - 1) if 0 <= r < x.shape[0]})
    biggest = torch.zeros((len(rows), n), dtype=torch.float64, device="cuda")
    for at in range(0, k, 8):
        biggest += (xv[rows, None, at:at + 8] * wv[None, :, at:at + 8]).abs().amax(-1)
    assert (err[rows] <= fine[rows] + 2.0 ** -10 * biggest).all(), float((err[rows] - fine[rows] - 2.0 ** -10 * biggest).max())


@pytest.mark.parametrize("dtype,rows,n,k,form", FORMS)
def test_each_form(dtype, rows, n, k, form):
    g = gen(rows + n + k)
    x, w = rows_of(rows, k, g), rows_of(n, k, g)
    assert form_of(x, w, DT[dtype]) == form
    out = run_linear(x, w, DT[dtype])
    check_linear(x, w, out)
    # the same bits again, and into strided rows at an odd place
    assert torch.equal(run_linear(x, w, DT[dtype]), out)
    room = torch.full((rows, n + 3), 5.0, dtype=DT[dtype], device="cuda")
    run_linear(x, w, DT[dtype], room[:, 1:1 + n])
    assert torch.equal(room[:, 1:1 + n], out) and (room[:, 0] == 5).all() and (room[:, 1 + n:] == 5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [33, 40])
def test_rows_and_weights_further_apart_than_tiles_reach(dtype, rows):
    n, k = 50, 1168
    x, w = rows_of(rows, k, gen(1)), rows_of(n, k, gen(2))
    def apart(m, stride):
        buf = torch.empty((m.shape[0], stride), dtype=torch.uint8, device="cuda")[:, 16:]
        return buf[:, :m._keep[0].shape[1]].copy_(m._keep[0]), m._keep[1]
    want = run_linear(x, w, DT[dtype])
    for a, b in ((blib.MX8(*apart(x, FAR)), w), (x, blib.MX8(*apart(w, FAR)))):
        assert form_of(a, b, DT[dtype]) == (STREAM, 2, 1, 4, 1)
        out = run_linear(a, b, DT[dtype])
        check_linear(x, w, out)
    assert form_of(x, w, DT[dtype])[0] == BATCH
    check_linear(x, w, want)


def shifted(x, w, g):
    """Scales of the groups of k moved by up to 100 in opposite directions: the
    same products."""
    d = torch.randint(-100, 101, ((x.shape[1] + 31) // 32,), generator=g).cuda()
    for m, by in ((x, d), (w, -d)):
        s = m._keep[1][:, :len(d)]
        s.copy_(s.int() + by)


@pytest.mark.parametrize("dtype,rows,n,k", [("bf16", *t[:3]) for t in TILES] + BATCHES)
def test_far_apart_scales_of_each_group(dtype, rows, n, k):
    g = gen(k)
    x, w = rows_of(rows, k, g), rows_of(n, k, g)
    shifted(x, w, g)
    s = torch.cat((x._keep[1][:, :k // 32].flatten(), w._keep[1][:, :k // 32].flatten()))
    assert s.min() < 30 and s.max() > 208 and s.max() < 248 and s.min() >= 10
    check_linear(x, w, run_linear(x, w, DT[dtype]))


@pytest.mark.parametrize("dtype,rows,n,k", [("bf16", *t[:3]) for t in TILES] + BATCHES)
def test_nan_stays_in_its_rows(dtype, rows, n, k):
    g = gen(n)
    x, w = rows_of(rows, k, g), rows_of(n, k, g)
    want = run_linear(x, w, DT[dtype]).clone()
    x._keep[1][1, 4] = 255
    x._keep[0][2, k - 15] = 0x7f
    w._keep[1][50, k // 32 - 1] = 255
    w._keep[0][n - 1, 0] = 0xff
    out = run_linear(x, w, DT[dtype])
    bad = torch.zeros((rows, n), dtype=torch.bool, device="cuda")
    bad[1], bad[2], bad[:, 50], bad[:, n - 1] = True, True, True, True
    assert out[bad].isnan().all() and torch.equal(out[~bad], want[~bad])


@pytest.mark.parametrize("dtype,rows,n,k", [("bf16", *t[:3]) for t in TILES] + BATCHES)
def test_what_lies_beside_the_rows_does_not_count(dtype, rows, n, k):
    """Rows apart, NaN codes around them and scale bytes behind the last group 255."""
    g = gen(rows)
    x, w = rows_of(rows, k, g), rows_of(n, k, g)
    groups, room = (k + 31) // 32, (k + 511) // 512 * 16
    def apart(m):
        codes = torch.full((m.shape[0] + 1, k + 48), 0x7f, dtype=torch.uint8, device="cuda")
        scales = torch.full((m.shape[0] + 1, room + 16), 255, dtype=torch.uint8, device="cuda")
        codes[:-1, 16:16 + k] = m._keep[0]
        scales[:-1, :groups] = m._keep[1][:, :groups]
        return blib.MX8(codes[:-1, 16:16 + k], scales[:-1, :room])
    a, b = apart(x), apart(w)
    assert form_of(a, b, DT[dtype]) == form_of(x, w, DT[dtype])
    assert torch.equal(run_linear(a, b, DT[dtype]), run_linear(x, w, DT[dtype]))


@pytest.mark.parametrize("dtype,rows,n,k", [("bf16", *t[:3]) for t in TILES] + BATCHES)
def test_one_workspace_captured_and_for_fewer_rows(dtype, rows, n, k):
    """A workspace of more rows, as an earlier call of another form left it; the
    call captured and replayed with eager work between."""
    dt, g = DT[dtype], gen(rows + k)
    most, w = rows_of(rows + 300, k, g), rows_of(n, k, g)
    x = most.rows(0, rows)
    want = run_linear(x, w, dt)
    ws = torch.full((blib.mx8_linear_workspace(most, w),), 255, dtype=torch.uint8, device="cuda")
    out, big = torch.zeros((rows, n), dtype=dt, device="cuda"), torch.zeros((rows + 300, n), dtype=dt, device="cuda")
    blib.mx8_linear(most, w, big, ws)
    blib.mx8_linear(x, w, out, ws)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        blib.mx8_linear(x, w, out, ws)
    for _ in range(4):
        out.fill_(7)
        blib.mx8_linear(most, w, big, ws)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("rows,form", [(16, STREAM), (255, BATCH), (255, TILE)])
@pytest.mark.parametrize("cx,cw", [(0x7e, 0x7e), (0x01, 0x01), (0x7e, 0x01), (0x38, 0xb8), (0x09, 0x5b), (0x78, 0x30)])
def test_one_product_of_every_pair_of_scales(rows, form, cx, cw):
    """Row i of x has scale i (of a few rows 17 i), row j of the weights scale j; one
    element of each is not 0.  bf16 outputs are the product, rounded once; fp32
    outputs that of the elements as they read back in bf16."""
    n, k = (255 if form != TILE else 25000), {STREAM: 64, BATCH: 96, TILE: 4096}[form]
    x, w = blib.MX8.empty(rows, k), blib.MX8.empty(n, k)
    step = 17 if rows == 16 else 1
    for m, c, by in ((x, cx, step), (w, cw, 1)):
        m._keep[0][:, 37] = c
        m._keep[1].copy_((by * torch.arange(m.shape[0], device="cuda") % 255).to(torch.uint8)[:, None].expand_as(m._keep[1]))
    assert form_of(x, w, torch.bfloat16)[0] == form
    # values from the bits, 2^(code - 127) too
    table = torch.cat((E4M3, torch.tensor([math.nan]), -E4M3, torch.tensor([math.nan]))).cuda()
    value = lambda m: table[m._keep[0][:, 37].int()] * (m._keep[1][:, 1].long() - 127 + 1023 << 52).view(torch.float64)
    want = value(x)[:, None] * value(w)                          # 8 bits: a bf16 number, unless below its normal range
    out = run_linear(x, w, torch.bfloat16)
    normal = want.abs() >= 2.0 ** -126
    assert torch.equal(out[normal].double(), want.bfloat16()[normal].double())
    assert ((out.double() - want).abs() <= 2.0 ** -133)[~normal].all()
    read = []
    for m in (x, w):
        t = torch.empty(m.shape, dtype=torch.bfloat16, device="cuda")
        blib.mx8_read(m, t)
        read.append(t[:, 37].double())
    want = read[0][:, None] * read[1]
    out = run_linear(x, w, torch.float32)
    same = (out == want.float()) | (out.isnan() & want.isnan()) | ((out.double() - want).abs() <= 2.0 ** -149)
    assert same.all()
