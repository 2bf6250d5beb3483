"""Attention over the paged 4-bit cache: page orders, both forms of the kernel
and what a call may need, beside test_kv4_gpu.py, whose plain implementation in
64 bits and tolerances these tests use."""
import pytest
import torch

from paper_2606_09514_amd import lib as blib
from test_kv4_gpu import CASES, DT, Setup, i32

pytestmark = pytest.mark.gpu


def run(s, parts, chunks=None, **bounds):
    """A call that has to take the form with so many parts of its weights (one:
    the prompt form), in so many chunks, checked with that form's tolerance."""
    max_rows, max_len = bounds.get("max_rows", max(s.news + [1])), bounds.get("max_len", max(s.lens))
    got = blib.kv4_attention_form(s.cache, s.dt, s.q.shape[1], s.n_rows, len(s.lens), max_rows, max_len)
    assert got[0] == parts and (chunks is None or chunks_are(got[1], chunks)), got
    s.call(**bounds)
    s.cols = 65 if parts == 1 else 1                           # what the tolerance goes by
    s.check()


def chunks_are(n, what):
    """One; few: joined by a wavefront or four for each row; many: by four."""
    return {"one": n == 1, "few": 1 < n <= 8, "many": n > 8}[what]


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


# ------------------------------------------------------------ the prompt form

PROMPTS = [
    # lens, new rows, query heads, KV heads, head_dim, page, chunks
    ([130], [71], 1, 1, 64, 16, "one"), ([68, 274], [68, 13], 1, 1, 64, 32, "one"), ([142], [17], 4, 1, 64, 64, "one"),
    ([162, 66], [14, 11], 16, 1, 64, 256, "one"), ([148, 103], [17, 20], 7, 1, 128, 16, "one"),
    ([147, 70], [8, 70], 1, 1, 128, 256, "one"), ([143, 112], [8, 15], 16, 1, 128, 128, "one"),
    ([300, 3, 0], [200, 9, 2], 16, 1, 128, 32, "one"), ([300, 0, 90], [200, 0, 9], 16, 1, 64, 16, "one"),
    ([1000, 900], [900, 300], 32, 8, 64, 64, "one"),
    # few (row, head) pairs to join (at most 4096), then more
    ([142, 1848, 173], [99, 13, 173], 14, 2, 64, 32, "few"), ([102, 253, 5646], [102, 253, 26], 8, 2, 128, 64, "few"),
    ([980, 240, 2341], [9, 240, 12], 16, 1, 64, 16, "few"), ([121, 5552, 376], [121, 16, 376], 8, 8, 64, 128, "few"),
    ([78, 340, 5935], [78, 340, 8], 12, 3, 128, 16, "few"), ([207, 3083, 325], [207, 10, 45], 16, 1, 128, 256, "few"),
    ([104, 98, 4027], [104, 98, 10], 16, 16, 64, 16, "many"), ([99, 510, 7767], [99, 510, 20], 4, 2, 128, 32, "many"),
    ([724, 7810, 250], [16, 8, 205], 14, 2, 128, 16, "many"),
]


@pytest.mark.parametrize("masked", [None, 0.5, 0.02], ids=["all", "half", "few"])
@pytest.mark.parametrize("case", range(len(PROMPTS)))
def test_prompt_form(case, masked):
    *sizes, chunks = PROMPTS[case]
    run(Setup(*sizes, torch.bfloat16, seed=case + 40, masked=masked), 1, chunks)


@pytest.mark.parametrize("masked", [None, 0.5], ids=["all", "half"])
def test_prompts_in_the_decode_form_keep_two_parts(masked):
    """bf16 calls of more than 64 columns that take the decode form, within the
    tolerance of its weights."""
    shapes = [c for c in CASES if max(c[1]) * (c[2] // c[3]) > 64] + [([2000], [600], 2, 2, 64, 64), ([700], [130], 8, 8, 64, 16),
                                                                      ([1500, 700, 90], [300, 200, 90], 7, 1, 128, 32)]
    taken = 0
    for i, c in enumerate(shapes):
        s = Setup(*c, torch.bfloat16, seed=i + 70, masked=masked)
        form = blib.kv4_attention_form(s.cache, s.dt, c[2], s.n_rows, len(c[0]), max(c[1]), max(c[0]))
        run(s, form[0])
        taken += form[0] == 2
    assert taken >= 4


@pytest.mark.parametrize("hd,page", [(64, 16), (64, 64), (128, 16), (128, 32), (128, 256)])
def test_prompt_form_pages_in_order(hd, page):
    for lens, news, nq, nkv in (([300, 90], [200, 9], 16, 1), ([102, 253, 5646], [102, 253, 26], 8, 2)):
        run(in_order(Setup(lens, news, nq, nkv, hd, page, torch.bfloat16, seed=page)), 1)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("chunks", ["one", "few"])
@pytest.mark.parametrize("page", [16, 64])
def test_prompt_form_sees_no_nan_it_may_not_see(page, chunks, hd):
    """NaN groups of values and keys, masked out, behind a row's own position
    or seen by some rows of a tile; every row of two sequences."""
    if chunks == "one":
        s = Setup([300, 90], [200, 9], 16, 1, hd, page, torch.bfloat16, seed=5, masked=0.9)
    else:
        s = Setup([207, 3083, 325], [207, 10, 45], 16, 1, hd, page, torch.bfloat16, seed=5, masked=0.9)
    ks, vs = s.cache._keep[2:]
    t, last = s.table.cpu(), [n - 1 for n in s.lens]
    groups = hd // 32
    # (sequence, position, scales, group, seen where not behind the row)
    for b, j, x, g, on in ((0, 50, vs, groups - 1, 0), (0, 150, vs, 0, 1), (0, 180, vs, groups - 1, 1), (0, 181, vs, 0, 1),
                           (0, 190, ks, 0, 1), (0, 120, ks, groups - 1, 0), (1, 20, vs, 0, 0), (1, last[1] - 4, vs, 1, 1),
                           (1, last[1] - 1, ks, groups - 1, 1), (1, 40, ks, 0, 0)):
        x[int(t[b, j // page]), 0, g, j % page] = 255
        s.mask[b, j] = on
    run(s, 1, chunks)
    nan = s.out[:s.cu_list[2]].cpu().isnan()
    first = s.lens[0] - s.news[0]                              # position of the first row
    assert not nan[:max(0, 150 - first)].any() and nan[max(0, 190 - first):s.news[0]].all()
    between = nan[max(0, 150 - first):190 - first]             # values only
    assert between[:, :, :32].all() and not between[:180 - max(150, first), :, 32:].any()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_prompt_form_leaves_out_pages_outside_the_pool(page, hd):
    for lens, news, chunks in (([300, 90], [200, 9], "one"), ([207, 3083, 325], [207, 10, 45], "few")):
        s = Setup(lens, news, 16, 1, hd, page, torch.bfloat16, seed=9, masked=0.9 if page == 32 else None)
        s.table[0, 0], s.table[1, 1], s.table[-1, 0] = -1, 2 ** 31 - 1, -2 ** 31
        if page <= 64:
            s.table[0, 2] = 10 ** 6
        run(s, 1, chunks)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("bounds,chunks", [((5, 3000), "few"), ((8, 2048), "few"), ((1000, 100000), "many")])
def test_prompt_form_bounds_that_differ_from_the_truth(bounds, chunks, hd):
    """More column tiles than the launch has workgroups for, longer sequences
    than it was split for, and a bound far above."""
    s = Setup([3000, 700, 5], [600, 40, 3], 16, 1, hd, 64, torch.bfloat16, seed=3)
    run(s, 1, chunks, max_rows=bounds[0], max_len=bounds[1])


def test_prompt_form_extremes_of_scale():
    for q_scale, scale in ((300.0, 1.0), (1e-6, 1.0), (1.0, 1e-30), (1.0, -2.0), (1.0, -0.1)):
        for lens, news in (([300, 90], [200, 9]), ([207, 3083, 325], [207, 10, 45])):
            s = Setup(lens, news, 16, 1, 128, 64, torch.bfloat16, seed=4, q_scale=q_scale)
            s.scale = scale
            if scale > 0:
                run(s, 1)
                continue
            s.call()
            want = s.out.clone()
            s.q, s.scale = -s.q, -scale                        # |scale| in the bounds
            s.out.fill_(5.0)
            run(s, 1)
            assert torch.equal(s.out, want)


# ------------------------------------------- one call's rows, others, replays


@pytest.mark.parametrize("dtype,lens,news,nq,nkv", [
    ("f32", [2100, 900, 33], [1, 1, 1], 8, 2), ("bf16", [2100, 900, 33], [1, 1, 1], 8, 2),
    ("f32", [300, 90], [200, 9], 16, 1), ("bf16", [300, 90], [200, 9], 16, 1),
    ("bf16", [207, 3083, 325], [207, 10, 45], 16, 1), ("bf16", [120011], [1], 32, 8),
    ("bf16", [3567, 2135, 5000], [763, 502, 1024], 4, 1)])
def test_equal_calls_give_equal_bits(dtype, lens, news, nq, nkv):
    s = Setup(lens, news, nq, nkv, 128, 64, DT[dtype], seed=8)
    a = s.call().clone()
    for _ in range(3):
        s.out.fill_(5.0)
        assert torch.equal(s.call(), a)


@pytest.mark.parametrize("dtype,lens,news,nq,nkv", [
    ("f32", [2100, 900, 33], [1, 1, 1], 8, 2), ("bf16", [2100, 900, 33], [1, 1, 1], 8, 2),
    ("f32", [300, 90], [40, 9], 16, 1), ("bf16", [162, 66], [14, 11], 16, 1)])
def test_a_sequence_alone_gives_the_bits_it_gives_among_others(dtype, lens, news, nq, nkv):
    """Where the form and the chunks, which the bounds of the call decide, are
    the same."""
    s = Setup(lens, news, nq, nkv, 128, 64, DT[dtype], seed=8)
    whole = s.call().clone()
    bounds = (max(news), max(lens))
    form = lambda B: blib.kv4_attention_form(s.cache, s.dt, nq, s.n_rows, B, *bounds)
    for b in range(len(lens)):
        assert form(1) == form(len(lens))
        n = blib.kv4_attention_workspace(s.cache, nq, s.n_rows, 1, *bounds)
        out = torch.full_like(s.out, 5.0)
        rows = slice(s.cu_list[b], s.cu_list[b + 1])
        blib.kv4_attention(s.cache, s.q, out, s.table[b:b + 1], s.len[b:b + 1], s.cu[b:b + 2], *bounds,
                           torch.full((n,), 255, dtype=torch.uint8, device="cuda"), scale=s.scale)
        assert torch.equal(out[rows], whole[rows])
        assert torch.all(out[:rows.start] == 5) and torch.all(out[rows.stop:] == 5)


def test_prompt_form_in_two_graphs():
    """Captured prompts replay with the lengths that the buffers then hold."""
    s = Setup([207, 3083, 325], [207, 10, 45], 16, 1, 128, 64, torch.bfloat16, seed=2)
    run(s, 1, "few")
    n = blib.kv4_attention_workspace(s.cache, 16, s.n_rows, 3, 207, 3083)
    works = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    graphs, outs = [], []
    for w in works:
        s.out = torch.full_like(s.out, 5.0)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.call(workspace=w)
        graphs.append(graph)
        outs.append(s.out)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for lens in ([207, 3083, 325], [207, 1500, 46], [0, 10, 300], [207, 3083, 325]):
        s.len.copy_(i32(lens))
        for o in outs:
            o.fill_(5.0)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1])
        s.lens, s.out, s.cols = lens, outs[0], 65
        s.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_workspace_for_a_batch_that_shrinks(dtype):
    """Requests end until one is left: in a buffer of the first step's rows, and
    in one of the rows that remain."""
    lens = [1300 - 7 * i for i in range(48)]
    s = Setup(lens, [1] * 48, 16, 4, 64, 32, DT[dtype], seed=12, extra_rows=0)
    work = torch.full((blib.kv4_attention_workspace(s.cache, 16, 48, 48, 1, 1300),), 255, dtype=torch.uint8, device="cuda")
    whole = (s.q, s.out)
    for B in (48, 16, 5, 1):
        s.lens, s.news, s.cu_list, s.cu = lens[:B], [1] * B, list(range(B + 1)), i32(list(range(B + 1)))
        s.table, s.len = s.table[:B].contiguous(), i32(lens[:B])
        for rows in (48, B):
            s.q, s.out, s.n_rows = whole[0][:rows], whole[1][:rows], rows
            s.out.fill_(5.0)
            s.call(workspace=work)
            s.check()


# ------------------------------------------------- weights of the prompt form


def rounded_bf16(x):
    return x.bfloat16().double()


def test_prompt_form_rounds_each_weight_once():
    """Four rows of a tile: D and A in its first half, C and B, above them by
    2^8 and more, in its second.  A's weight is in bf16 by the time that C moves
    the maximum.  out = (p_A v - p_B v) / sum of p with v = 6 * 2^9, where A and
    B almost cancel, shows their errors: each at most e = 2^-8, plus 2^-19 for
    scores below 32 in fp32 (their rounding and exp2's).  So
    |do| <= e sum_j p_j |v_j - out| / (sum p (1 - e)), and the output's own
    rounding.  The queries are those of many for which a second rounding of A's
    weight, behind its product with the maximum's move, would pass that bound."""
    hd, row = 64, dict(D=2, A=3, C=40, B=41)
    ln2 = torch.tensor(2.0).log().item()
    g = torch.Generator().manual_seed(1)
    n = 400000
    rnd = lambda lo, hi: lo + (hi - lo) * torch.rand(n, generator=g, dtype=torch.float64)
    # scores in units of log2, each the sum of two bf16 numbers
    d = rnd(0, 1)
    want_s = dict(D=d, A=d - rnd(0, 3), C=d + rnd(8.5, 9.5), B=None)
    q = {}
    for r in "DAC":
        q[r] = torch.stack([rounded_bf16(want_s[r]), rounded_bf16(want_s[r] - rounded_bf16(want_s[r]))])
    near = q["A"].sum(0) + rnd(-0.01, 0.01)                    # p_B close to p_A
    q["B"] = torch.stack([rounded_bf16(near), rounded_bf16(near - rounded_bf16(near))])
    s = {r: q[r].sum(0) for r in q}
    v = dict(D=0.0, A=6 * 2.0 ** 9, C=0.0, B=-6 * 2.0 ** 9)

    def out_of(p):
        return sum(p[r] * v[r] for r in p) / sum(p.values())

    p = {r: torch.exp2(s[r] - s["C"]) for r in s}
    want, e = out_of(p), 2.0 ** -8 + 2.0 ** -19
    bound = e * sum(p[r] * (v[r] - want).abs() for r in p) / (sum(p.values()) * (1 - e))
    twice = {r: rounded_bf16(p[r]) for r in p}
    for r in "DA":
        twice[r] = rounded_bf16(rounded_bf16(torch.exp2(s[r] - s["D"])) * torch.exp2(s["D"] - s["C"]))
    over = ((out_of(twice) - want).abs() - 2.0 ** -8 * want.abs()) / bound
    pick = over.topk(128).indices
    assert over[pick].min() > 1.1

    S = Setup([143], [8], 16, 1, hd, 64, torch.bfloat16, seed=1, masked=0.5, extra_rows=0)
    k, vv, ks, vs = S.cache._keep
    S.mask.zero_()
    for i, r in enumerate("DACB"):
        pg, at = int(S.table[0, row[r] // 64]), row[r] % 64
        S.mask[0, row[r]] = 1
        k[pg, 0, at] = 0
        k[pg, 0, at, i] = 0x22                                 # 1 and 1 at elements 2 i, 2 i + 1
        ks[pg, 0, :, at] = 127
        vv[pg, 0, at] = {0.0: 0, 1.0: 0x77, -1.0: 0xff}[(v[r] > 0) - (v[r] < 0) + 0.0]
        vs[pg, 0, :, at] = 127 + 9
    S.q.zero_()
    x = torch.stack([t for r in "DACB" for t in q[r]], -1)[pick]          # [128][8]
    S.q[:, :, :8] = x.view(8, 16, 8).bfloat16().cuda()
    S.scale = torch.tensor(ln2).item()
    run(S, 1, "one")
    got = S.out.cpu().double().view(128, hd)
    assert torch.equal(got, got[:, :1].expand(-1, hd))
    err = (got[:, 0] - want[pick]).abs() - 2.0 ** -8 * got[:, 0].abs()
    assert torch.all(err <= bound[pick]), float((err / bound[pick]).max())


# ----------------------------------------------------- other calls it allows


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,news", [([300, 90], [1, 1]), ([300, 90], [200, 9])], ids=["tokens", "prompt"])
def test_queries_that_are_not_finite_stay_in_their_rows(lens, news, dtype):
    s = Setup(lens, news, 16, 1, 128, 64, DT[dtype], seed=21)
    s.q[0, 3, 5] = float("nan")
    s.q[-4, 7, 100] = float("inf")
    s.call()
    s.check()
    assert s.out[0, 3].isnan().all() and s.out[s.cu_list[-1] - 1, 7].isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_thousand_sequences(dtype):
    """Sequences of no rows, one and several among them; column tiles times
    sequences past what a launch's dimension starts with."""
    g = torch.Generator().manual_seed(9)
    lens = torch.randint(0, 70, (1001,), generator=g).tolist()
    news = [min(int(n), 9) if i % 3 else min(int(n), 1) for i, n in enumerate(lens)]
    s = Setup(lens, news, 4, 1, 64, 16, DT[dtype], seed=22)
    s.call()
    s.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 64])
def test_sequences_that_share_pages(page, dtype):
    """Three sequences whose first rows are the same pages, one of which has a
    page twice."""
    s = Setup([300, 280, 220], [1, 3, 2], 8, 1, 64, page, DT[dtype], seed=23)
    shared = 192 // page
    s.table[1:, :shared] = s.table[0, :shared]
    s.table[2, 1] = s.table[2, 0]
    s.call()
    s.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_step_as_two_calls_over_its_sequences(dtype):
    """Prompts and single tokens as calls of their own, the queries and outputs
    whole: each writes its rows and no others."""
    s = Setup([300, 90, 700, 33, 1200], [200, 9, 1, 1, 1], 16, 1, 64, 16, DT[dtype], seed=24)
    for lo, hi in ((2, 5), (0, 2)):
        bounds = (max(s.news[lo:hi]), max(s.lens[lo:hi]))
        n = blib.kv4_attention_workspace(s.cache, 16, s.n_rows, hi - lo, *bounds)
        before = s.out.clone()
        blib.kv4_attention(s.cache, s.q, s.out, s.table[lo:hi], s.len[lo:hi], s.cu[lo:hi + 1], *bounds,
                           torch.full((n,), 255, dtype=torch.uint8, device="cuda"), scale=s.scale)
        for rows in (slice(0, s.cu_list[lo]), slice(s.cu_list[hi], None)):
            assert torch.equal(s.out[rows], before[rows])
    s.cols = 65                                                # one part for the prompts' calls of bf16
    s.check()
