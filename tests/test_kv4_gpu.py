"""Serving from the paged 4-bit cache on the device, each entry point against
a plain implementation in 64 bits (or whole numbers) on the host side of
torch, at the sizes and masks where it can go wrong, and a run of them
together.

Tolerances.  Page planning and the 4-bit values of finished rows are exact.
u = 2^-24 is an fp32 rounding (relative), r the output type's: bf16 2^-8, fp32
u.

Norm and rotation, x (of a pair x, y) before: the sum of head_dim squares
takes at most 12 roundings in a row and its mean, eps, root and reciprocal 5,
of which the square root halves the first 14: 7 + 3 = 10 u; two products 2 u;
cos and sin are within 3 u (angles and series are fp64, rounded once: 1 u and
a little); a product each and their sum:
less than 16 u (|x| + |y|) in all, and one output rounding r |result|.

Attention.  s = scale q . k: products exact in fp32 at most u off each, summed
in at most head_dim + 4 additions, then scaled: |ds| <= (head_dim + 8) u
scale sum |q k|.  A weight exp(s - m): relative error ds (its own and the
maximum's: 2 ds) plus 4 u of exp2 and its argument's rounding (in ds' bound),
plus the split into bf16 parts (2^-16 with two, u with three, 2^-8 with one,
whose rounding the denominator shares: the same 2 (..) bound).  Sums over n
rows: at most n / 32 + 32 additions of fp32 in a row, in numerator and
denominator.  So |do| <= (2 (2 ds + 4 u + split) + 2 (n / 32 + 40) u) sum p |v| /
sum p, and one output rounding."""
import math

import pytest
import torch

from paper_2606_09514_amd import lib as blib

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: U}

def split(dt, cols):
    """Rounding of a softmax weight: two bf16 parts, three in fp32 calls; one
    where a bf16 call has more than 64 columns (query heads of a KV head times
    rows)."""
    return U if dt is torch.float32 else 2.0 ** -8 if cols > 64 else 2.0 ** -16


E2M1 = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------ 4-bit format


def scale_exponent(amax):
    """Least e with amax <= 7 * 2^e, within -125..125 (64-bit amax > 0)."""
    e = torch.floor(torch.log2(amax.clamp(min=1e-300))) - 3
    for _ in range(3):
        e = torch.where(amax > 7 * torch.exp2(e), e + 1, e)
    return e.clamp(-125, 125)


def quantised(x):
    """Finite values [..., hd] as the cache holds them, in 64 bits."""
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    e = scale_exponent(g.abs().amax(-1, keepdim=True))
    a = g / torch.exp2(e)
    d = (a.unsqueeze(-1).abs() - E2M1[:8]).abs()
    best = d.amin(-1, keepdim=True)
    # nearest; of two, the one with an even code
    pick = torch.where(d == best, torch.tensor([0, 2, 0, 2, 0, 2, 0, 2]) + 1, 100).argmin(-1)
    return (torch.sign(a) * E2M1[pick] * torch.exp2(e)).reshape(x.shape)


def cache_values(cache):
    """The four tensors of a cache -> K, V [pages][n_kv][rows][hd], 64 bits, host."""
    out = []
    for codes, scales in ((0, 2), (1, 3)):
        c, s = cache._keep[codes].cpu().long(), cache._keep[scales].cpu()
        x = E2M1[torch.stack((c & 15, c >> 4), -1).flatten(-2)]
        sv = torch.exp2(s.double() - 127)
        sv[s == 255] = math.nan
        out.append(x * sv.transpose(-1, -2).repeat_interleave(32, -1))
    return out


def random_cache(pages, page, nkv, hd, seed, junk=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = blib.KV4.empty(pages, page, nkv, hd)
    for t in c._keep[:2]:
        t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    for t in c._keep[2:]:
        t.copy_(torch.randint(124, 129, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    return c


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,nkv,page", [(128, 8, 64), (64, 2, 16), (128, 1, 256), (64, 5, 128), (128, 3, 32)])
def test_append_and_read(dtype, hd, nkv, page):
    dt = DT[dtype]
    g = torch.Generator().manual_seed(hd + nkv + page)
    n, pages = 37, 9
    # rows of a wider projection; magnitudes from 2^-40 to 2^40, ties and the
    # border amax = 7 * 2^e among them
    qkv = torch.randn((n, 3 * nkv, hd), generator=g)
    qkv *= torch.exp2(torch.randint(-40, 41, (n, 3 * nkv, hd // 32), generator=g).float()).repeat_interleave(32, -1)
    qkv[3, nkv:, :32] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7] * 4)
    qkv[4, nkv:, :32] = torch.tensor([7.03125, -7.03125, 0, -0.25] * 8)
    qkv[5, nkv:] = 0
    qkv[6, nkv:, :] = torch.tensor([3.38e38, -1e38, 1e-38, 1.0]).repeat(hd // 4)
    qkv = qkv.to(dt).cuda()
    k, v = qkv[:, nkv:2 * nkv], qkv[:, 2 * nkv:]
    slots = torch.randperm(pages * page, generator=g)[:n].to(torch.int32)
    slots[7], slots[8] = -1, pages * page                      # not in the pool: not written
    slots[9] = 2 ** 31 - 1
    cache = blib.KV4.empty(pages, page, nkv, hd)
    before = [t.clone() for t in cache._keep]
    blib.kv4_append(cache, k, v, slots.cuda())
    K, V = cache_values(cache)
    live = [i for i in range(n) if 0 <= slots[i] < pages * page]
    for x, got in ((k, K), (v, V)):
        want = quantised(x.cpu())
        for i in live:
            s = int(slots[i])
            assert torch.equal(got[s // page, :, s % page], want[i]), i
    # nothing else of the pool changed
    rows = torch.ones(pages * page, dtype=torch.bool)
    rows[slots[live].long()] = False
    for t, b in zip(cache._keep[:2], before[:2]):
        a, b = (z.cpu().transpose(1, 2).reshape(pages * page, -1)[rows] for z in (t, b))
        assert torch.equal(a, b)
    for out_dt in (torch.bfloat16, torch.float32):
        ko = torch.full((n, nkv, hd), 9.0, dtype=out_dt, device="cuda")
        vo = torch.full((n, nkv + 1, hd), 9.0, dtype=out_dt, device="cuda")[:, 1:]
        blib.kv4_read(cache, slots.cuda(), ko, vo)
        for x, got in ((K, ko), (V, vo)):
            for i in range(n):
                s = int(slots[i])
                want = x[s // page, :, s % page] if i in live else torch.full((nkv, hd), 9.0, dtype=torch.float64)
                assert torch.equal(got[i].cpu().double(), want), i


def test_append_makes_groups_of_infinities_and_nan_nan():
    cache = blib.KV4.empty(2, 16, 2, 64)
    k = torch.ones((3, 2, 64), device="cuda")
    v = torch.ones((3, 2, 64), device="cuda")
    k[0, 0, 5], k[1, 1, 40], v[2, 0, 63] = math.inf, math.nan, -math.inf
    blib.kv4_append(cache, k, v, i32([0, 17, 31]))
    K, V = cache_values(cache)
    bad = torch.zeros((3, 2, 2), dtype=torch.bool)
    for s, i in ((0, 0), (17, 1), (31, 2)):
        for x, src in ((K, k), (V, v)):
            got = x[s // 16, :, s % 16].reshape(2, 2, 32)
            fine = src[i].cpu().reshape(2, 2, 32).isfinite().all(-1)
            assert torch.equal(got.isnan().all(-1), ~fine) and torch.equal(got.isnan().any(-1), ~fine)
            assert torch.all(got[fine] == 1)
    ko = torch.zeros((1, 2, 64), device="cuda")
    vo = torch.zeros((1, 2, 64), device="cuda", dtype=torch.float32)
    blib.kv4_read(cache, i32([0]), ko, vo)
    assert ko[0, 0, :32].isnan().all() and torch.all(ko[0, 0, 32:] == 1) and torch.all(vo == 1)


# ------------------------------------------------------- norm and rotation


def rotated(x, w, pos, theta, d, inter, eps):
    """64-bit norm and rotation, and |x| + |y| of each element's pair."""
    x = x.double().cpu()
    if w is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w.double().cpu()
    i = torch.arange(d // 2, dtype=torch.float64)
    ang = pos.double().cpu()[:, None, None] * theta ** (-2 * i / d) if d else torch.zeros((len(pos), 1, 0)).double()
    a, b = (slice(0, d, 2), slice(1, d, 2)) if inter else (slice(0, d // 2), slice(d // 2, d))
    y, mag = x.clone(), x.abs()
    y[..., a] = x[..., a] * ang.cos() - x[..., b] * ang.sin()
    y[..., b] = x[..., b] * ang.cos() + x[..., a] * ang.sin()
    mag[..., a] = mag[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, mag


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,nq,nkv,hd,part,inter,norm", [
    (1, 32, 8, 128, 1.0, False, "qk"), (5, 4, 2, 64, 1.0, False, "qk"), (3, 28, 4, 128, 0.5, False, "q"),
    (19, 7, 7, 64, 0.25, True, "k"), (33, 1, 1, 128, 1.0, True, ""), (9, 5, 3, 64, 0.0, False, "qk"),
    (700, 40, 40, 128, 0.25, False, ""), (130, 3, 1, 64, 0.5, True, "qk")])
def test_qk_norm_rope(dtype, n, nq, nkv, hd, part, inter, norm):
    dt = DT[dtype]
    g = torch.Generator().manual_seed(n + nq)
    qkv = torch.randn((n, nq + 2 * nkv, hd), generator=g).to(dt).cuda()
    q, k = qkv[:, :nq], qkv[:, nq:nq + nkv]
    w = {s: (1 + 0.2 * torch.randn(hd, generator=g)).to(dt).cuda() if s in norm else None for s in "qk"}
    pos = torch.randint(0, 1 << 20, (n,), generator=g).to(torch.int32)
    pos[0] = 0
    if n > 4:
        pos[2] = -1                                            # left as it was
    d = int(hd * part)
    outs = [torch.full((n, h + 1, hd), 7.0, dtype=dt, device="cuda")[:, 1:] for h in (nq, nkv)]
    kw = dict(q_norm=w["q"], k_norm=w["k"], eps=1e-5, theta=5e5, rope_dim=d, interleaved=inter)
    blib.qk_norm_rope(q, k, pos.cuda(), *outs, **kw)
    for x, side, got in ((q, "q", outs[0]), (k, "k", outs[1])):
        want, mag = rotated(x, w[side], pos, 5e5, d, inter, 1e-5)
        err = (got.cpu().double() - want).abs()
        tol = 16 * U * mag + ROUND[dt] * want.abs() * (1 + 16 * U) + 1e-37
        live = pos >= 0
        assert torch.all(err[live] <= tol[live]), float((err[live] / tol[live]).max())
        assert torch.all(got.cpu()[~live] == 7)
    # in place
    q2, k2 = q.clone(), k.clone()
    blib.qk_norm_rope(q2, k2, pos.cuda(), q2, k2, **kw)
    live = (pos >= 0).cuda()
    assert torch.equal(q2[live], outs[0][live]) and torch.equal(k2[live], outs[1][live])
    assert torch.equal(q2[~live], q[~live])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,nq,nkv,hd,page,norm", [(1, 32, 8, 128, 64, True), (6, 4, 2, 64, 16, False),
                                                   (41, 40, 40, 128, 32, True), (300, 7, 1, 128, 256, True),
                                                   (17, 6, 3, 64, 128, True)])
def test_append_qkv(dtype, n, nq, nkv, hd, page, norm):
    """Queries and values as the separate calls give them, bit for bit; keys
    within half a 4-bit step of the 64-bit ones."""
    dt = DT[dtype]
    g = torch.Generator().manual_seed(n)
    qkv = torch.randn((n, nq + 2 * nkv, hd), generator=g).to(dt).cuda()
    q, k, v = qkv[:, :nq], qkv[:, nq:nq + nkv], qkv[:, nq + nkv:]
    w = [(1 + 0.2 * torch.randn(hd, generator=g)).to(dt).cuda() if norm else None for _ in range(2)]
    pos = torch.randint(0, 50000, (n,), generator=g).to(torch.int32)
    pages = -(-n // page) + 2
    slots = torch.randperm(pages * page, generator=g)[:n].to(torch.int32)
    if n > 4:
        pos[1], slots[3] = -1, -1
    cache, plain = blib.KV4.empty(pages, page, nkv, hd), blib.KV4.empty(pages, page, nkv, hd)
    q_out, q_sep = torch.full_like(q, 3.0), torch.full_like(q, 3.0)
    k_sep = torch.zeros_like(k)
    kw = dict(q_norm=w[0], k_norm=w[1], theta=1e6)
    blib.kv4_append_qkv(cache, q, k, v, pos.cuda(), slots.cuda(), q_out, **kw)
    blib.qk_norm_rope(q, k, pos.cuda(), q_sep, k_sep, **kw)
    slots2 = torch.where(pos < 0, -1, slots)
    blib.kv4_append(plain, k_sep, v, slots2.to(torch.int32).cuda())
    assert torch.equal(q_out, q_sep)
    assert torch.equal(cache._keep[1], plain._keep[1]) and torch.equal(cache._keep[3], plain._keep[3])
    if dt is torch.float32:                                    # nothing is rounded between
        assert torch.equal(cache._keep[0], plain._keep[0]) and torch.equal(cache._keep[2], plain._keep[2])
    want, mag = rotated(k, w[1], pos, 1e6, hd, False, 1e-6)
    K, _ = cache_values(cache)
    for i in range(n):
        s = int(slots2[i])
        if s < 0:
            continue
        x, off = want[i].reshape(nkv, -1, 32), (16 * U * mag[i]).reshape(nkv, -1, 32)
        got = K[s // page, :, s % page].reshape(nkv, -1, 32)
        step = torch.exp2(scale_exponent((x.abs() + off).amax(-1, keepdim=True)))
        assert torch.all((got - x).abs() <= torch.maximum(step / 4, x.abs() / 4) + 2 * off), i


def test_norm_of_tiny_zero_and_huge_rows():
    """Means of squares that are subnormal, zero (with and without eps), near
    the largest number and past it, in fp32."""
    for eps in (0.0, 1e-6):
        q = torch.zeros((5, 1, 64), device="cuda")
        q[0], q[1, 0, 0], q[2], q[3], q[4] = 3e-20, 2.0, 0.0, 1.5e19, 1e30
        k, pos = q.clone(), i32([0] * 5)
        w = torch.full((64,), 0.5, device="cuda")
        blib.qk_norm_rope(q, k, pos, q, k, q_norm=w, eps=eps)
        got = q.cpu().double()
        # squares, a tree of sums, eps, root, two products: 16 roundings, and
        # subnormal squares off by 2^-150 each
        m = (torch.tensor(3e-20, dtype=torch.float32).double() ** 2)
        off = 16 * U + 2.0 ** -150 / (m.item() + eps)
        want = 0.5 * 3e-20 / math.sqrt(m.item() + eps)
        assert torch.all((got[0] - want).abs() <= off * want + 2.0 ** -149)
        want = 0.5 * 2 / math.sqrt(4 / 64 + eps)
        assert abs(got[1, 0, 0].item() - want) <= 16 * U * want and torch.all(got[1, 0, 1:] == 0)
        assert torch.all(got[2] == 0) if eps else got[2].isnan().all()
        assert torch.all(got[3:] == 0)                         # the sum, or each square, overflows: 1 / sqrt(inf)
        assert torch.all(k[3] == q.new_tensor(1.5e19)) and torch.all(k[4] == q.new_tensor(1e30))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_as_a_few_at_a_time(dtype):
    """Thousands of rows, several workgroups' worth for every CU, bit for bit
    as calls of single rows and of odd pieces give them."""
    dt, n, nq, nkv, hd, page = DT[dtype], 9001, 3, 2, 64, 64
    g = torch.Generator().manual_seed(11)
    qkv = torch.randn((n, nq + 2 * nkv, hd), generator=g).to(dt).cuda()
    q, k, v = qkv[:, :nq], qkv[:, nq:nq + nkv], qkv[:, nq + nkv:]
    pos = torch.randint(-2000, 100000, (n,), generator=g).to(torch.int32).cuda()
    pages = -(-n // page)
    slots = torch.randperm(pages * page, generator=g)[:n].to(torch.int32).cuda()
    w = [(1 + 0.2 * torch.randn(hd, generator=g)).to(dt).cuda() for _ in range(2)]
    whole, parts = blib.KV4.empty(pages, page, nkv, hd), blib.KV4.empty(pages, page, nkv, hd)
    plain, plain_parts = blib.KV4.empty(pages, page, nkv, hd), blib.KV4.empty(pages, page, nkv, hd)
    outs = [torch.full((n, h, hd), 5.0, dtype=dt, device="cuda") for h in (nq, nq, nq, nkv, nq, nkv)]
    cuts = [0, 1, 2, 7, 1000, 1001, 5000, n]
    for lo, hi, cache, a in [(0, n, whole, 0)] + [(*c, parts, 1) for c in zip(cuts, cuts[1:])]:
        c = slice(lo, hi)
        blib.kv4_append_qkv(cache, q[c], k[c], v[c], pos[c], slots[c], outs[a][c], q_norm=w[0], k_norm=w[1])
        blib.qk_norm_rope(q[c], k[c], pos[c], outs[2 + 2 * a][c], outs[3 + 2 * a][c], q_norm=w[0], k_norm=w[1])
        blib.kv4_append((plain, plain_parts)[a], k[c], v[c], slots[c])
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[2], outs[4]) and torch.equal(outs[3], outs[5])
    assert torch.equal(outs[0], outs[2]) and torch.all(outs[0][pos < 0] == 5)
    for a, b in ((whole, parts), (plain, plain_parts)):
        for x, y in zip(a._keep, b._keep):
            assert torch.equal(x, y)
    assert not torch.equal(whole._keep[0], plain._keep[0])
    got = [torch.zeros((n, nkv, hd), dtype=dt, device="cuda") for _ in range(2)]
    blib.kv4_read(plain, slots, *got)
    for x, y in zip(got, (k, v)):
        for i in (0, 1, 4096, n - 1):
            assert torch.equal(x[i].cpu().double(), quantised(y[i].cpu()))


# ---------------------------------------------------------------- planning


def plan_reference(lens, news, page, table, ring, state, n_rows):
    """What buddy_plan_pages documents, request after request."""
    B, cols = len(table), len(table[0])
    head, count = state
    table = [list(t) for t in table]
    asked_pages = asked_rows = taken = rows = 0
    len_out, cu, pos, slots, refused = [], [0], [], [], []
    up = lambda x: -(-x // page)
    for b in range(B):
        n, f = lens[b], news[b]
        why = 0
        if n < 0 or f < 0 or n + f > cols * page:
            why = 1
        else:
            need = up(n + f) - up(n)
            asked_pages += need
            asked_rows += f
            if need > 0 and asked_pages > count:
                why = 2
            elif f > 0 and asked_rows > n_rows:
                why = 3
        refused.append(why)
        if why:
            len_out.append(max(n, 0))
            cu.append(rows)
            continue
        for i in range(need):
            table[b][up(n) + i] = ring[(head + taken) % len(ring)]
            taken += 1
        for p in range(n, n + f):
            pos.append(p)
            slots.append(table[b][p // page] * page + p % page)
        rows += f
        len_out.append(n + f)
        cu.append(rows)
    pad = [-1] * (n_rows - rows)
    return table, [(head + taken) % len(ring), count - taken], len_out, cu, pos + pad, slots + pad, refused


def run_plan(lens, news, page, table, ring, state, n_rows, alias=False):
    B = len(lens)
    d = dict(len=i32(lens), new=i32(news), table=i32(table), ring=i32(ring), state=i32(state))
    out = dict(state=d["state"] if alias else i32([-5, -5]), len=d["len"] if alias else i32([-5] * B),
               cu=i32([-5] * (B + 1)), pos=i32([-5] * n_rows), slots=i32([-5] * n_rows),
               refused=torch.full((B,), 9, dtype=torch.uint8, device="cuda"))
    blib.plan_pages(d["len"], d["new"], d["table"], d["ring"], d["state"], page, out["state"], out["len"], out["cu"],
                    out["pos"], out["slots"], out["refused"])
    return (d["table"].tolist(), out["state"].tolist(), out["len"].tolist(), out["cu"].tolist(), out["pos"].tolist(),
            out["slots"].tolist(), out["refused"].tolist())


@pytest.mark.parametrize("B,page,free,n_rows,new,kind", [
    (1, 16, 10, 16, 5, "even"), (1, 64, 0, 8, 1, "even"), (7, 32, 40, 300, 60, "ragged"), (256, 64, 300, 256, 1, "even"),
    (257, 16, 90, 1100, 4, "ragged"), (1000, 128, 900, 5000, 9, "ragged"), (1024, 256, 2000, 20000, 40, "ragged"),
    (64, 16, 37, 4000, 30, "few pages"), (64, 32, 4000, 333, 30, "few rows"), (40, 64, 50, 500, 30, "bad lengths"),
    (12, 16, 600, 9000, 700, "prompts")])
@pytest.mark.parametrize("alias", [False, True])
def test_plan_pages(B, page, free, n_rows, new, kind, alias):
    g = torch.Generator().manual_seed(B + page)
    rnd = lambda hi, n=B: torch.randint(0, hi, (n,), generator=g).tolist()
    lens = rnd(5 * page) if kind != "prompts" else [0] * B
    news = rnd(new + 1) if kind != "even" else [new] * B
    cols = 5 + (new + page - 1) // page
    if kind == "bad lengths":
        lens[3], news[5], lens[9], news[9], lens[11] = -4, -1, 2 ** 31 - 1, 2 ** 31 - 1, cols * page + 1
    held = [max(0, min(cols, -(-n // page))) for n in lens]
    total = sum(held) + free
    ids = torch.randperm(max(total, 1), generator=g).tolist()
    table, at = [], 0
    for h in held:
        table.append(ids[at:at + h] + [-77] * (cols - h))
        at += h
    ring, head = [-99] * max(total, 1), total // 3
    for i in range(free):
        ring[(head + i) % total] = ids[at + i]
    got = run_plan(lens, news, page, table, ring, [head, free], n_rows, alias)
    want = plan_reference(lens, news, page, table, ring, [head, free], n_rows)
    for a, b, what in zip(got, want, ("table", "state", "len", "cu", "pos", "slots", "refused")):
        assert list(a) == list(b), what
    why = {"few pages": 2, "few rows": 3, "bad lengths": 1}.get(kind)
    assert why is None or why in got[6]


@pytest.mark.parametrize("B,n_rows", [(5, 100), (5, 30000), (600, 30000)])
def test_plan_in_place_in_part(B, n_rows):
    """Only the state or only the lengths written in place, and neither: the
    same plan."""
    g = torch.Generator().manual_seed(B)
    page, cols = 32, 210 if B == 5 else 4
    lens, news = torch.randint(0, 60, (B,), generator=g).tolist(), torch.randint(0, n_rows // B, (B,), generator=g).tolist()
    held = [-(-n // page) for n in lens]
    total = sum(held) + B * cols
    ids = torch.randperm(total, generator=g).tolist()
    table, at = [], 0
    for h in held:
        table.append(ids[at:at + h] + [-77] * (cols - h))
        at += h
    want = plan_reference(lens, news, page, table, ids[at:] + ids[:at], [total - 3, total - at], n_rows)
    for state_too, len_too in ((0, 0), (1, 0), (0, 1), (1, 1)):
        d = dict(len=i32(lens), state=i32([total - 3, total - at]), table=i32(table))
        state_out, len_out = d["state"] if state_too else i32([0, 0]), d["len"] if len_too else i32([0] * B)
        cu, pos, slots = i32([0] * (B + 1)), i32([0] * n_rows), i32([0] * n_rows)
        refused = torch.full((B,), 9, dtype=torch.uint8, device="cuda")
        blib.plan_pages(d["len"], i32(news), d["table"], i32(ids[at:] + ids[:at]), d["state"], page, state_out, len_out, cu,
                        pos, slots, refused)
        for a, b in zip((d["table"], state_out, len_out, cu, pos, slots, refused), want):
            assert a.tolist() == [list(r) if isinstance(r, tuple) else r for r in b]


def test_plan_keeps_within_a_damaged_ring_and_table():
    """A ring state and ids that no call of the library wrote: every access
    stays inside the arrays, and bad ids become slots of -1."""
    got = run_plan([20, 3], [40, 2], 16, [[7, -3, 5, 9], [1000000, 1, 1, 1]], [12345, -8, 2], [-7, 99], 64)
    # head -7 is entry 2 of three; count 99 is 3 of three; request 0 takes two
    assert got[0][0] == [7, -3, 2, 12345] and got[1] == [1, 1]
    assert got[2] == [60, 5] and got[6] == [0, 0]
    slots = [-1] * 12 + [2 * 16 + i for i in range(16)] + [-1] * 12 + [-1] * 2
    assert got[5] == slots + [-1] * 22


@pytest.mark.parametrize("B,page", [(1, 16), (5, 64), (300, 32), (1024, 16)])
@pytest.mark.parametrize("alias", [False, True])
def test_release_pages(B, page, alias):
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 6 * page, (B,), generator=g).tolist()
    done = (torch.rand(B, generator=g) < 0.5).tolist()
    if B > 100:
        lens[7], lens[8], done[7], done[8] = -3, 100 * page, True, True
    cols = 6
    held = [-(-n // page) if 0 <= n <= cols * page else 0 for n in lens]
    pages = sum(held) + 9
    ids = torch.randperm(pages, generator=g).tolist()
    table, at = [], 0
    for h in held:
        table.append(ids[at:at + h] + [-1] * (cols - h))
        at += h
    head = pages - 4
    ring = [-99] * pages
    for i in range(9):
        ring[(head + i) % pages] = ids[at + i]
    want, tail = list(ring), head + 9
    for b in range(B):
        if done[b]:
            for i in range(held[b]):
                want[tail % pages] = table[b][i]
                tail += 1
    d = dict(len=i32(lens), ring=i32(ring), state=i32([head, 9]))
    so, lo = (d["state"], d["len"]) if alias else (i32([0, 0]), i32([0] * B))
    blib.release_pages(d["len"], torch.tensor(done, dtype=torch.uint8, device="cuda"), i32(table), d["ring"],
                       d["state"], page, so, lo)
    assert d["ring"].tolist() == want and so.tolist() == [head, tail - head]
    assert lo.tolist() == [0 if e else n for n, e in zip(lens, done)]


# --------------------------------------------------------------- attention


class Setup:
    """Sequences over a shuffled pool, whose unused pages and rows behind the
    sequences' ends are NaN."""

    def __init__(self, lens, news, nq, nkv, hd, page, dt, seed, masked=None, extra_rows=3, q_scale=1.5):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.news, self.page, self.dt, self.hd = list(lens), list(news), page, dt, hd
        held = [-(-n // page) for n in lens]
        pages = sum(held) + 4
        self.cache = random_cache(pages, page, nkv, hd, seed)
        ids = torch.randperm(pages, generator=g).to(torch.int32)
        cols = max(held + [1]) + 1
        table, at = torch.full((len(lens), cols), pages + 9, dtype=torch.int32), 0
        used = torch.zeros((pages, page), dtype=torch.bool)
        for b, h in enumerate(held):
            table[b, :h] = ids[at:at + h]
            for i in range(h):
                used[ids[at + i], :max(0, lens[b] - i * page)] = True
            at += h
        for t in self.cache._keep[2:]:
            t.masked_fill_(~used.cuda()[:, None, None, :], 255)
        self.table = table.cuda()
        cu = [0]
        for n in news:
            cu.append(cu[-1] + n)
        self.cu_list, self.cu = cu, i32(cu)
        self.n_rows = cu[-1] + extra_rows
        self.len = i32(lens)
        # a view of a wider buffer, rows apart
        self.q = (q_scale * torch.randn((self.n_rows, nq + 2, hd), generator=g)).to(dt).cuda()[:, 1:nq + 1]
        self.out = torch.full((self.n_rows, nq + 1, hd), 5.0, dtype=dt, device="cuda")[:, :nq]
        self.mask = None
        if masked is not None:
            self.mask = (torch.rand((len(lens), max(lens) + 5), generator=g) < masked).to(torch.uint8).cuda()
        self.scale = hd ** -0.5

    def call(self, max_rows=None, max_len=None, workspace=None, stream=None):
        max_rows = max(self.news + [1]) if max_rows is None else max_rows
        max_len = max(self.lens) if max_len is None else max_len
        if workspace is None:
            n = blib.kv4_attention_workspace(self.cache, self.q.shape[1], self.n_rows, len(self.lens), max_rows, max_len)
            workspace = torch.full((n,), 255, dtype=torch.uint8, device="cuda")     # NaN to whoever reads it first
        self.cols = max_rows * (self.q.shape[1] // self.cache.shape[0])
        blib.kv4_attention(self.cache, self.q, self.out, self.table, self.len, self.cu, max_rows, max_len, workspace,
                           mask=self.mask, scale=self.scale, stream=stream)
        return self.out

    def check(self):
        K, V = cache_values(self.cache)
        pages, nkv = K.shape[:2]
        nq = self.q.shape[1]
        G, hd, page = nq // nkv, self.hd, self.page
        out, q, table = self.out.cpu().double(), self.q.cpu().double(), self.table.cpu()
        mask = None if self.mask is None else self.mask.cpu()
        for b, (n, f) in enumerate(zip(self.lens, self.news)):
            if f == 0:
                continue
            n = min(n, table.shape[1] * page)
            j = torch.arange(n)
            ids = table[b].long()[j // page]
            ok = (ids >= 0) & (ids < pages)
            if mask is not None:
                on = torch.zeros(n, dtype=torch.bool)
                w = min(n, mask.shape[1])
                on[:w] = mask[b, :w] != 0
                ok = ok & on
            ids = torch.where((ids >= 0) & (ids < pages), ids, 0)
            rows = slice(self.cu_list[b], self.cu_list[b + 1])
            see = ok & (j <= (n - f + torch.arange(f))[:, None])          # [f][n]
            for h in range(nq):
                k, v = K[ids, h // G, j % page], V[ids, h // G, j % page]
                k = torch.where(ok[:, None], k, 0.0)
                qh = q[rows, h]
                s = qh @ k.T * self.scale
                ds = (hd + 8) * U * self.scale * (qh.abs() @ k.abs().T)
                s = s.masked_fill(~see, -math.inf)
                p = torch.softmax(s, -1) if n else s
                p = torch.where(see.any(-1, keepdim=True), p, 0.0)
                nan_v = v.isnan()
                v0 = torch.where(nan_v, 0.0, v)
                want = p @ v0
                want = torch.where((see.double() @ nan_v.double()) > 0, math.nan, want)
                dmax = torch.where(see, ds, 0.0).amax(-1, keepdim=True) if n else torch.zeros((f, 1)).double()
                part = 2 * (2 * dmax + 4 * U + split(self.dt, self.cols)) + 2 * (n / 32 + 40) * U
                tol = part * (p @ v0.abs()) + ROUND[self.dt] * (want.abs() * (1 + part)) + 1e-30
                got = out[rows, h]
                assert torch.equal(got.isnan(), want.isnan()), (b, h)
                err = torch.where(want.isnan(), 0.0, (got - want).abs())
                tol = torch.where(want.isnan(), 1.0, tol)
                assert torch.all(err <= tol), (b, h, float((err / tol).max()))
        assert torch.all(self.out[self.cu_list[-1]:] == 5)                 # rows behind the last sequence


CASES = [
    # lens, new rows, query heads, KV heads, head_dim, page
    ([1], [1], 32, 8, 128, 64), ([2], [2], 4, 2, 64, 16), ([31, 32, 33], [1, 1, 1], 8, 2, 128, 16),
    ([2048], [1], 8, 2, 128, 64), ([5000], [1], 4, 1, 128, 128), ([777, 1, 64, 130], [1] * 4, 7, 1, 128, 32),
    ([100, 300, 17, 260, 64], [1, 1, 0, 1, 1], 3, 3, 64, 64), ([0, 40, 0], [1, 1, 0], 16, 1, 128, 16),
    ([640], [5], 16, 1, 64, 32), ([90, 256], [7, 3], 6, 2, 128, 16), ([200], [200], 4, 1, 128, 64),
    ([513, 70], [130, 70], 8, 2, 128, 256), ([300, 5, 129], [33, 5, 64], 4, 4, 64, 16), ([3], [9], 4, 2, 128, 16),
    ([1500] * 20, [1] * 20, 8, 8, 128, 64), ([9000], [3], 2, 2, 64, 256),
]


@pytest.mark.parametrize("masked", [None, 0.5, 0.02], ids=["all", "half", "few"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case, dtype, masked):
    s = Setup(*CASES[case], DT[dtype], seed=case + 1, masked=masked)
    s.call()
    s.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_sees_no_nan_it_may_not_see(dtype):
    """NaN rows masked out, behind a token's own position, or seen: only what
    is seen, and only in the group of elements that is NaN (values) or
    everywhere (keys)."""
    for news in ([1, 1], [40, 9], [200, 9]):
        s = Setup([300, 90], news, 4, 1, 128, 32, DT[dtype], seed=5, masked=0.9)
        k, v, ks, vs = s.cache._keep
        t = s.table.cpu()
        place = lambda b, j: (int(t[b, j // 32]), j % 32)
        for b, j, mask in ((0, 50, 0), (0, 295, 1), (0, 280, 1), (1, 20, 0), (1, 85, 1)):
            pg, r = place(b, j)
            vs[pg, 0, 2, r] = 255
            s.mask[b, j] = mask
        pg, r = place(0, 290)
        ks[pg, 0, 1, r] = 255
        s.mask[0, 290] = 1
        pg, r = place(1, 40)
        ks[pg, 0, 0, r] = 255
        s.mask[1, 40] = 0
        s.call()
        K, _ = cache_values(s.cache)
        # a NaN key that is seen makes the whole row NaN
        want_nan = torch.zeros((s.cu_list[-1], 4), dtype=torch.bool)
        for i in range(news[0]):
            want_nan[i] = 300 - news[0] + i >= 290
        got = s.out[:s.cu_list[-1]].cpu()
        assert torch.all(got[want_nan].isnan())
        s_rows = [i for i in range(s.cu_list[-1]) if not want_nan[i, 0]]
        for i in s_rows:
            b = 0 if i < news[0] else 1
            p = (300 - news[0] + i) if b == 0 else 90 - news[1] + (i - news[0])
            seen = (p >= 280) if b == 0 else p >= 85
            nan = got[i].isnan()
            assert torch.all(nan[:, 64:96] == seen) and not nan[:, :64].any() and not nan[:, 96:].any(), (i, p)


def test_attention_leaves_out_pages_outside_the_pool():
    for page, news in ((16, [1, 1]), (64, [1, 1]), (32, [100, 3])):
        s = Setup([400, 100], news, 8, 2, 128, page, torch.float32, seed=9)
        s.table[0, 1], s.table[0, 3], s.table[1, 0] = -1, 2 ** 31 - 1, -2 ** 31
        if page == 64:
            s.table[1, 1] = 10 ** 6                            # nothing of the sequence is left
        s.call()
        s.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_bounds_below_the_truth_cost_no_rows(dtype):
    s = Setup([3000, 700, 5], [40, 1, 3], 8, 2, 128, 64, DT[dtype], seed=3)
    s.call(max_rows=1, max_len=100)
    s.check()
    s.out.fill_(5.0)
    s.call(max_rows=1000, max_len=100000)
    s.check()


def test_attention_extremes_of_scale():
    """Scores far apart, nearly equal ones, tiny and negative scales."""
    for q_scale, scale in ((300.0, 1.0), (1e-6, 1.0), (1.0, 1e-30), (1.0, -2.0), (1.0, -0.1)):
        s = Setup([1000, 50], [1, 20], 4, 1, 128, 64, torch.float32, seed=4, q_scale=q_scale)
        s.scale = scale
        s.call()
        if scale < 0:                                          # |scale| in the bounds
            s.q, s.scale = -s.q, -scale
        s.check()
    s = Setup([600, 90], [100, 20], 4, 1, 128, 64, torch.bfloat16, seed=4)   # the prompt form
    s.scale = -0.2
    s.call()
    s.q, s.scale = -s.q, 0.2
    s.check()


def test_attention_offsets_past_32_bits():
    pages, page = 40000, 256                                   # 5.2 GB of codes a side
    c = blib.KV4.empty(pages, page, 8, 128)
    s = Setup([600], [1], 16, 8, 128, page, torch.bfloat16, seed=6)
    far = [pages - 1, 39000, 35000]
    for big, small in zip(c._keep, s.cache._keep):
        for i, p in enumerate(far):
            big[p] = small[int(s.table[0, i])]
    s.call()
    want = s.out.clone()
    s.cache, s.table = c, i32([far + [0]])
    s.out.fill_(5.0)
    s.call()
    assert torch.equal(s.out, want)
    slots = i32([far[0] * page + 7, far[2] * page + 80])
    k = torch.randn((2, 8, 128), device="cuda")
    ko, vo = torch.zeros_like(k), torch.zeros_like(k)
    blib.kv4_append(c, k, -k, slots)
    blib.kv4_read(c, slots, ko, vo)
    assert torch.equal(ko.cpu().double(), quantised(k.cpu())) and torch.equal(vo, -ko)


def test_attention_repeats_bit_for_bit_and_alone():
    """Equal calls give equal bits; a sequence does not depend on the others
    where the chunks are the same (the bounds of the call decide them)."""
    s = Setup([2100, 900, 33], [1, 1, 1], 8, 2, 128, 64, torch.float32, seed=8)
    a = s.call().clone()
    s.out.fill_(5.0)
    assert torch.equal(s.call(), a)


def test_one_stream_and_another_and_two_graphs():
    """Calls enqueued on the stream they are given; captured steps replay with
    the lengths the buffers then hold, two graphs with a workspace each."""
    s = Setup([700, 300], [1, 1], 8, 2, 128, 64, torch.bfloat16, seed=2)
    want = s.call().clone()
    n = blib.kv4_attention_workspace(s.cache, 8, s.n_rows, 2, 1, 700)
    works = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    side = torch.cuda.Stream()
    s.out.fill_(5.0)
    side.wait_stream(torch.cuda.current_stream())
    s.call(workspace=works[0], stream=side)
    side.synchronize()
    assert torch.equal(s.out, want)
    graphs, outs = [], []
    for w in works:
        s.out = torch.full_like(s.out, 5.0)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.call(workspace=w)
        graphs.append(graph)
        outs.append(s.out)
    for lens in ([700, 300], [650, 1], [12, 280], [700, 300]):
        s.len.copy_(i32(lens))
        for o in outs:
            o.fill_(5.0)
        torch.cuda.synchronize()
        s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
        with torch.cuda.stream(s1):
            graphs[0].replay()
        with torch.cuda.stream(s2):
            graphs[1].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1])
        s.lens, s.out = lens, outs[0]
        s.check()


def test_refusals_on_the_device_write_nothing():
    s = Setup([64], [1], 4, 2, 64, 16, torch.float32, seed=1)
    w = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    args = (s.cache, s.q, s.out, s.table, s.len, s.cu, 1, 64)
    assert blib.kv4_attention(*args, w[:8], check=False) == blib.EINVAL
    assert blib.kv4_attention(*args, w, scale=math.inf, check=False) == blib.EINVAL
    assert blib.kv4_attention(*args[:-1], 70, w, mask=torch.ones((1, 69), dtype=torch.uint8, device="cuda"),
                              check=False) == blib.EINVAL
    odd = torch.zeros((3, 4, 65), device="cuda")[:, :, 1:]
    with pytest.raises(ValueError, match="contiguous"):
        blib.kv4_attention(s.cache, odd, *args[2:], w)
    with pytest.raises(TypeError, match="int32"):
        blib.kv4_attention(*args[:4], s.len.long(), *args[5:], w)
    with pytest.raises(ValueError, match="cu_rows"):
        blib.kv4_attention(*args[:5], s.len, *args[6:], w)
    with pytest.raises(blib.BuddyError):
        blib.qk_norm_rope(s.q, s.q[:, :2], i32([0] * s.n_rows), s.out, s.out[:, :2].clone(), rope_dim=24)
    half = torch.zeros((3, 4, 64), device="cuda", dtype=torch.float16)
    with pytest.raises(TypeError):
        blib.kv4_append(s.cache, half[:, :2], half[:, :2], s.cu)
    torch.cuda.synchronize()
    assert torch.all(s.out == 5)


# ------------------------------------------------------------ all together


@pytest.mark.parametrize("captured", [False, True], ids=["eager", "graph"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_serving_steps(dtype, captured):
    """Prompts admitted, single tokens, a request that ends and a new one in
    its place: release, plan, then a layer's append and attention each step,
    against 64-bit attention over the values that the cache should hold."""
    dt, nq, nkv, hd, page, B, cols, rows = DT[dtype], 6, 2, 64, 16, 4, 8, 64
    g = torch.Generator().manual_seed(7)
    pages = 22
    cache = blib.KV4.empty(pages, page, nkv, hd)
    for t in cache._keep[2:]:
        t.fill_(255)                                           # pages of nobody: NaN
    ring = torch.randperm(pages, generator=g).to(torch.int32).cuda()
    st = dict(len=i32([0] * B), new=i32([0] * B), done=torch.zeros(B, dtype=torch.uint8, device="cuda"),
              table=i32([[-1] * cols] * B), state=i32([5, pages]), cu=i32([0] * (B + 1)), pos=i32([0] * rows),
              slots=i32([0] * rows), refused=torch.zeros(B, dtype=torch.uint8, device="cuda"))
    qkv = torch.zeros((rows, nq + 2 * nkv, hd), dtype=dt, device="cuda")
    q, k, v = qkv[:, :nq], qkv[:, nq:nq + nkv], qkv[:, nq + nkv:]
    q_out, out = torch.zeros((rows, nq, hd), dtype=dt, device="cuda"), torch.zeros((rows, nq, hd), dtype=dt, device="cuda")
    w = [(1 + 0.2 * torch.randn(hd, generator=g)).to(dt).cuda() for _ in range(2)]
    work = torch.zeros(blib.kv4_attention_workspace(cache, nq, rows, B, rows, cols * page), dtype=torch.uint8, device="cuda")

    def step():
        blib.release_pages(st["len"], st["done"], st["table"], ring, st["state"], page, st["state"], st["len"])
        blib.plan_pages(st["len"], st["new"], st["table"], ring, st["state"], page, st["state"], st["len"], st["cu"],
                        st["pos"], st["slots"], st["refused"])
        blib.kv4_append_qkv(cache, q, k, v, st["pos"], st["slots"], q_out, q_norm=w[0], k_norm=w[1])
        blib.kv4_attention(cache, q_out, out, st["table"], st["len"], st["cu"], rows, cols * page, work)

    graph = None
    if captured:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            step()
    held, hist = [0] * B, [([], []) for _ in range(B)]
    steps = [([30, 1, 0, 17], []), ([1, 1, 20, 1], []), ([1, 1, 1, 1], []), ([40, 0, 1, 1], [0]), ([1, 1, 1, 1], [1]),
             ([1, 50, 1, 1], []), ([1, 1, 1, 1], []), ([5, 1, 1, 1], [2, 3])]
    for news, ended in steps:
        qkv.copy_(torch.randn(qkv.shape, generator=g).to(dt))
        q_out.fill_(5.0)
        out.fill_(5.0)
        st["new"].copy_(i32(news))
        st["done"].copy_(torch.tensor([b in ended for b in range(B)], dtype=torch.uint8))
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        assert not st["refused"].any()
        for b in ended:
            held[b], hist[b] = 0, ([], [])
        K, V = cache_values(cache)
        pos, slots, at = st["pos"].tolist(), st["slots"].tolist(), 0
        assert st["state"][1].item() == pages - sum(-(-(h + n) // page) for h, n in zip(held, news))
        for b, n in enumerate(news):
            first = at
            for i in range(n):
                assert pos[at] == held[b] + i
                hist[b][0].append(K[slots[at] // page, :, slots[at] % page])
                hist[b][1].append(V[slots[at] // page, :, slots[at] % page])
                want = quantised(v[at].cpu())
                assert torch.equal(hist[b][1][-1], want)
                at += 1
            held[b] += n
            if n == 0:
                continue
            kk, vv = torch.stack(hist[b][0]), torch.stack(hist[b][1])      # [len][n_kv][hd]
            for h in range(nq):
                kh, vh = kk[:, h // 3], vv[:, h // 3]
                qh = q_out[first:at, h].cpu().double()
                s = qh @ kh.T / 8
                see = torch.arange(held[b]) <= (held[b] - n + torch.arange(n))[:, None]
                p = torch.softmax(s.masked_fill(~see, -math.inf), -1)
                ds = ((hd + 8) * U / 8 * (qh.abs() @ kh.abs().T)).amax(-1, keepdim=True)
                part = 2 * (2 * ds + 4 * U + split(dt, 3 * rows)) + 2 * (held[b] / 32 + 40) * U
                want = p @ vh
                tol = part * (p @ vh.abs()) + ROUND[dt] * want.abs() * (1 + part) + 1e-30
                assert torch.all((out[first:at, h].cpu().double() - want).abs() <= tol), (b, h)
        assert torch.all(out[at:] == 5) and torch.all(q_out[at:] == 5) and pos[at:] == [-1] * (rows - at)
