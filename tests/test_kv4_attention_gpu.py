"""Attention over the paged 4-bit cache: page orders, both forms of the kernel
and what a call may need, beside test_kv4_gpu.py, whose plain implementation in
64 bits and tolerances these tests use."""
import pytest
import torch

from test_kv4_gpu import DT, Setup

pytestmark = pytest.mark.gpu


def in_order(s):
    """The same sequences with their pages one after the other in the pool, as
    a fresh ring hands them out."""
    pages = s.cache._keep[0].shape[0]
    table = s.table.cpu()
    used = [int(p) for row in table for p in row if 0 <= p < pages]
    order = torch.tensor(used + [p for p in range(pages) if p not in set(used)]).cuda()
    for t in s.cache._keep:
        t.copy_(t[order].clone())
    at = 0
    for row in table:
        for i, p in enumerate(row.tolist()):
            if 0 <= p < pages:
                row[i], at = at, at + 1
    s.table.copy_(table)
    return s


@pytest.mark.parametrize("masked", [None, 0.5], ids=["all", "half"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nkv,page", [(1, 16), (2, 16), (1, 32)])
def test_pages_one_after_the_other(nkv, page, hd, dtype, masked):
    """Two neighbours of 16 rows share a slab: with one KV head the second's
    codes follow the first's, its scales do not."""
    for lens, news in (([100, 47, 16, 333], [1, 1, 1, 1]), ([200, 33], [5, 3])):
        s = in_order(Setup(lens, news, 2 * nkv, nkv, hd, page, DT[dtype], seed=hd + page, masked=masked))
        assert s.table[0, 1] == s.table[0, 0] + 1
        s.call()
        s.check()


def test_largest_scales():
    """The largest scale that a call takes, of either sign, over scores of a few
    tens."""
    for news in ([1, 1], [20, 3]):
        s = Setup([300, 90], news, 8, 2, 128, 64, torch.float32, seed=11, q_scale=5e-31)
        s.scale = 1e30
        s.call()
        s.check()
        s.q, want = -s.q, s.out.clone()
        s.out.fill_(5.0)
        s.scale = -1e30
        assert torch.equal(s.call(), want)
