"""The operators around attention at the ends of their ranges, on the device:
rows that one workgroup takes one behind another, with padding among them; sums
in place; adapters of many rows and outputs; sampling at low temperatures."""
import math

import pytest
import torch

from paper_2606_09514_amd import lib as blib
from test_serving_gpu import DT, ROUND, U, adapters_of, check_sample, gen, mx8_of, run_linear, run_lora, values

pytestmark = pytest.mark.gpu


def test_norm_of_three_rows_a_workgroup_with_padding_between():
    """Rows 2^20 apart are one workgroup's: a live one, padding and a live one,
    and other patterns, two wavefronts a row.  Live rows have the bits that they
    have alone, padding stays."""
    step, width = 2 ** 20, 640
    n = 3 * step + 5
    pattern = torch.randint(-40, 41, (61, width), generator=gen(1)).cuda()         # row r: pattern r % 61, times 2^(r % 7)
    r = torch.arange(n, device="cuda")
    h = torch.empty((n, width), dtype=torch.bfloat16, device="cuda")
    for at in range(0, n, step):
        part = r[at:at + step]
        h[at:at + step] = pattern[part % 61] * torch.exp2((part % 7).float())[:, None]
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    pos[step:2 * step] = -1                                      # live, padding, live
    pos[:1000], pos[step + 500:step + 2000], pos[2 * step + 800:2 * step + 2500] = -1, 0, -1   # the other patterns
    w = (1 + 0.2 * torch.randn(width, generator=gen(2))).bfloat16().cuda()
    y = torch.full((n, width), 9.0, dtype=torch.bfloat16, device="cuda")
    blib.add_rmsnorm(h, w, y=y, pos=pos)
    one = torch.empty((61 * 7, width), dtype=torch.bfloat16, device="cuda")       # every row that there is: r % 427
    blib.add_rmsnorm(h[:427].contiguous(), w, y=one)
    for at in range(0, n, step):
        part, live = r[at:at + step], pos[at:at + step, None] >= 0
        assert torch.equal(y[at:at + step], torch.where(live, one[part % 427], 9.0))


@pytest.mark.parametrize("hidden", [torch.float32, torch.bfloat16])
def test_norm_in_place_keeps_the_rows_where_they_are(hidden):
    g = gen(3)
    buf = torch.randn((7, 80), generator=g).to(hidden).cuda()
    before = buf.clone()
    h, apart = buf[:, :64], buf.view(-1)[:560].as_strided((7, 64), (72 if hidden is torch.float32 else 64, 1))
    delta, w = torch.randn((7, 64), generator=g).bfloat16().cuda(), torch.ones(64, dtype=torch.bfloat16, device="cuda")
    y = torch.full_like(delta, 9.0)
    with pytest.raises(blib.BuddyError):
        blib.add_rmsnorm(h, w, delta=delta, h_out=apart, y=y)
    assert torch.equal(buf, before) and (y == 9).all()
    want, want_y = torch.empty((7, 64), dtype=hidden, device="cuda"), torch.empty_like(delta)
    blib.add_rmsnorm(h, w, delta=delta, h_out=want, y=want_y)
    blib.add_rmsnorm(h, w, delta=delta, h_out=h, y=y)
    assert torch.equal(h, want) and torch.equal(y, want_y) and torch.equal(buf[:, 64:], before[:, 64:])
    blib.add_rmsnorm(before[2:3, :64], w, delta=delta[2:3], h_out=before[2:3, :64].as_strided((1, 64), (64, 1)), y=y[:1])   # a row has no stride
    assert torch.equal(before[2, :64], want[2]) and torch.equal(y[0], want_y[2])


# rows, adapters, rank, d_in, d_out: tiles of 64 rows with ranks up to 16, 32, 64
# and 128, of 16 rows too, and 1, 2, 4 and 8 blocks of outputs a workgroup
# (pieces of tiles times blocks of 256 outputs: from 4096, 8192 and 16384 on)
MANY = [(1100, 2, 16, 520, 264), (1100, 2, 24, 520, 264), (1500, 3, 32, 264, 1032), (1025, 1, 64, 520, 61448), (1300, 1, 128, 264, 65288),
        (1100, 1, 32, 136, 61192), (2100, 1, 56, 264, 61448), (2100, 1, 8, 264, 65288), (4099, 1, 40, 136, 65288), (1000, 1, 32, 136, 16520),
        (1000, 5, 128, 72, 36104), (1000, 3, 40, 72, 65288)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n,rank,k,d", MANY)
def test_adapters_of_many_outputs(dtype, rows, n, rank, k, d):
    """The tolerance of the adapters' own test (t of fp32 adapters is not split), the
    reference on the device in 64 bits, an adapter at a time; in place as well."""
    dt, g = DT[dtype], gen(rows + d)
    ad = adapters_of(n, rank, k, d, dt, rows)
    x = torch.randn((rows, k), generator=g).to(dt).cuda()
    y = torch.randn((rows, d + 8), generator=g).to(dt).cuda()[:, :d]
    ids = torch.randint(-1, n, (rows,), generator=g)
    ids[[3, rows - 1]] = torch.tensor([-2, n])
    out = torch.full((rows, d + 8), 9.0, dtype=dt, device="cuda")
    run_lora(ad, x, y, out[:, :d], ids.tolist())
    assert (out[:, d:] == 9).all()
    for i in range(-2, n + 1):
        at = (ids == i).nonzero()[:, 0].cuda()
        if not 0 <= i < n:
            assert torch.equal(out[at, :d], y[at] if i == -1 else torch.full_like(y[at], 9.0))
            continue
        a, b, s = ad._keep[0][i].double(), ad._keep[1][i].double().T.contiguous(), ad._keep[2][i].double()
        xv, yv = x[at].double(), y[at].double()
        t, dtv = xv @ a.T.contiguous(), (k + 16) * U * (xv.abs() @ a.T.abs().contiguous())
        add = s * (t @ b)
        tol = s * ((dtv + (2.0 ** -16 if dtype == "bf16" else 0) * t.abs()) @ b.abs() + (rank + 16) * U * (t.abs() @ b.abs()))
        tol += 4 * U * (yv.abs() + add.abs()) + ROUND[dt] * (yv + add).abs()
        err = (out[at, :d].double() - yv - add).abs()
        assert (err <= tol).all(), float((err - tol).max())
    y2 = y.clone()
    run_lora(ad, x, y2, y2, ids.tolist())
    live = ((ids >= -1) & (ids < n)).cuda()
    assert torch.equal(y2, torch.where(live[:, None], out[:, :d], y))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,v", [(1, 50021), (30, 9001), (3, 151001)])
def test_sampling_at_low_temperatures(dtype, b, v):
    """A top_k that reaches behind the last token with a weight: no token of weight
    0 is drawn, whichever are listed on the way."""
    g = gen(v)
    x = (2 * torch.randn((b, v), generator=g)).to(DT[dtype])
    x[:, ::17] = -math.inf
    x = x.cuda()
    u = torch.rand(b, generator=g).tolist()
    u[0] = 0.99999994
    for t in (0.02, 0.1, 0.3):
        for k in (1, 20, 50, 1000, 6000):
            check_sample(x, u, [t] * b, [k] * b)
            check_sample(x, u, [t] * b, [k] * b, [0.95] * b)
        check_sample(x, u, [t] * b, [1000] * b, [0.9] * b, [0.01] * b)
        check_sample(x, u, [t] * b, p=[0.9] * b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_projection_of_the_most_rows(dtype):
    """2^20 rows of x, 2^20 weight rows, and outputs past 2^31 elements, each against
    calls of a part of the rows."""
    dt = DT[dtype]
    eight = lambda rows, k, seed: mx8_of(torch.randn((rows, k), device="cuda", generator=torch.Generator("cuda").manual_seed(seed)))
    for rows, n, k in ((2 ** 20, 40, 144), (2 ** 20, 24, 128), (9, 2 ** 20, 256), (40, 2 ** 20, 128), (140000, 16400, 128)):
        x, w = eight(rows, k, 1), eight(n, k, 2)
        out = run_linear(x, w, dt)
        for r in {0, rows // 2, max(rows - 300, 0)}:
            for c in {0, n // 2, max(n - 520, 0)}:
                part, cols = x.rows(r, min(r + 300, rows)), w.rows(c, min(c + 520, n))
                xv, wv = values(part).cuda(), values(cols).cuda()
                want, total = xv @ wv.T.contiguous(), xv.abs() @ wv.T.abs().contiguous()
                tol = (k + 16) * U * total if dtype == "f32" else (2.0 ** -10 + (k / 8 + 64) * U) * total   # sum of maxima <= sum |p|
                assert ((out[r:r + 300, c:c + 520].double() - want).abs() <= tol + ROUND[dt] * want.abs()).all(), (rows, n, k, r, c)
        assert not out.isnan().any()
        del out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,k,d", [(3, 16, 16), (4096, 8, 24), (2, 8, 2056)])
def test_adapters_of_the_most_rows(dtype, n, k, d):
    """2^20 rows, of few and of the most adapters, and outputs past 2^31 elements."""
    dt, rows, rank = DT[dtype], 2 ** 20, 8
    ad = adapters_of(n, rank, k, d, dt, n)
    x = torch.randn((rows, k), device="cuda").to(dt)
    y = torch.randn((rows, d), device="cuda").to(dt)
    ids = torch.randint(-2, n + 1, (rows,), dtype=torch.int32, device="cuda")
    ids[:5000] = 0                                               # a long run
    plan = torch.empty(blib.lora_plan_size(rows, n), dtype=torch.int32, device="cuda")
    ws = torch.empty(blib.lora_workspace(ad, rows), dtype=torch.uint8, device="cuda")
    out = torch.full_like(y, 9.0)
    blib.lora_plan(ids, n, plan)
    blib.lora_add(ad, x, y, out, plan, ws)
    a, b, s = (t.double() for t in ad._keep)
    for at in range(0, rows, 2 ** 16):
        p = slice(at, at + 2 ** 16)
        i = ids[p].long()
        live, j = (i >= 0) & (i < n), i.clamp(0, n - 1)
        xv, yv = x[p].double(), y[p].double()
        t, size = (a[j] * xv[:, None]).sum(-1), (a[j] * xv[:, None]).abs().sum(-1)
        add, tol = torch.zeros_like(yv), torch.zeros_like(yv)
        for q in range(rank):                                    # the adapters' own tolerance
            bq = b[:, :, q].contiguous()[j]
            add += t[:, q:q + 1] * bq
            tol += ((k + 16) * U * size[:, q:q + 1] + (2.0 ** -16 + (rank + 16) * U) * t[:, q:q + 1].abs()) * bq.abs()
        add, tol = s[j][:, None] * add, s[j][:, None] * tol
        want = torch.where(live[:, None], yv + add, torch.where(i[:, None] == -1, yv, torch.tensor(9.0, dtype=torch.float64, device="cuda")))
        tol = torch.where(live[:, None], tol + 4 * U * (yv.abs() + add.abs()) + ROUND[dt] * want.abs(), 0.0)
        assert ((out[p].double() - want).abs() <= tol).all(), at


def test_sampling_of_the_largest_rows_and_batches():
    g = gen(9)
    v = 2 ** 20
    x = torch.randn((4, v + 1), generator=g)
    x[0] = 1.5                                                   # every token the same
    x[1, : v // 2] = -math.inf
    for t in (torch.float32, torch.bfloat16):
        l = x.to(t).cuda()[:, 1:]
        u = [0.99999994, 0.0, 0.5, 0.25]
        check_sample(l, u, [1.0] * 4)
        check_sample(l, u, [0.7] * 4, [v - 1, v, v // 3, 5000], [0.999, 0.5, 0.9, 1.0])
        check_sample(l, u, [1.3] * 4, p=[0.99999994, 0.9, 0.1, 0.5], m=[0.5, 0.0, 0.1, 0.02])
    b = 65535
    l = torch.tensor([1.0, 3.0, 2.0]).repeat(b, 1)
    l[torch.arange(b), torch.randint(0, 3, (b,), generator=g)] = -math.inf
    token, ws = torch.full((b,), -9, dtype=torch.int32, device="cuda"), torch.empty(blib.sample_workspace(b, 3), dtype=torch.uint8, device="cuda")
    f = lambda c: torch.full((b,), c, device="cuda")
    blib.sample(l.cuda(), f(0.5), token, ws, f(0.0))
    assert torch.equal(token.cpu().long(), l.argmax(1))
    blib.sample(l.cuda(), f(0.9999), token, ws, f(5.0), top_p=f(0.999))   # two tokens each, both kept
    assert torch.equal(token.cpu(), torch.where(l[:, 2] > 0, 2, 1).int())
