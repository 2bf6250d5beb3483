"""The operators around attention at the ends of their ranges, on the device:
rows that one workgroup takes one behind another, with padding among them; sums
in place."""
import pytest
import torch

from paper_2606_09514_amd import lib as blib
from test_serving_gpu import gen

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
