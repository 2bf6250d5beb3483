"""The operators around attention as a server uses them, on the device: steps
of a whole block over the paged cache, eager and captured; given streams, two
captured graphs at once, workspaces of more rows, rows far apart, no rows, and
what the binding refuses.  Tolerances are those of the operators' own tests,
applied to the values that each operator of a step was given."""
import pytest
import torch

from paper_2606_09514_amd import lib as blib
from test_serving_gpu import (DT, ROUND, U, adapters_of, gen, i32, linear_case, linear_tolerance, lora_reference, mx8_of, near_8bit,
                              run_linear, run_lora, token_of, values)

pytestmark = pytest.mark.gpu

B, COLS, ROWS, PAGE, PAGES = 4, 8, 64, 16, 26
NQ, NKV, HD, D, FF, VOCAB = 6, 2, 64, 256, 688, 1003
ADAPTERS = 3


class Served:
    """A block's weights, a step's buffers and a server's state."""

    def __init__(self, dtype):
        g = gen(11)
        self.dt = dt = dtype
        matrix = lambda n, k: mx8_of((torch.randn((n, k), generator=g) / k ** 0.5).cuda())
        self.w = dict(qkv=matrix((NQ + 2 * NKV) * HD, D), o=matrix(D, NQ * HD), gu=matrix(2 * FF, D), down=matrix(D, FF),
                      head=matrix(VOCAB, D))
        weight = lambda n: (1 + 0.2 * torch.randn(n, generator=g)).to(dt).cuda()
        self.norms, self.head_norms = [weight(D) for _ in range(3)], [weight(HD) for _ in range(2)]
        self.ad = adapters_of(ADAPTERS, 16, D, (NQ + 2 * NKV) * HD, dt, 5)
        self.cache = blib.KV4.empty(PAGES, PAGE, NKV, HD)
        self.ring = torch.randperm(PAGES, generator=g).to(torch.int32).cuda()
        u8 = lambda n: torch.zeros(n, dtype=torch.uint8, device="cuda")
        self.len, self.new, self.done, self.table = i32([0] * B), i32([0] * B), u8(B), i32([[-1] * COLS] * B)
        self.state, self.cu, self.pos, self.slots, self.refused = i32([0, PAGES]), i32([0] * (B + 1)), i32([0] * ROWS), i32([0] * ROWS), u8(B)
        self.ids = i32([-2] * ROWS)
        z = lambda n, t=dt: torch.zeros((ROWS, n), dtype=t, device="cuda")
        self.h = z(D, torch.float32)
        self.y, self.a, self.a2, self.a3 = z(D), *(blib.MX8.empty(ROWS, D) for _ in range(3))
        self.qkv_y, self.qkv, self.q, self.att = z((NQ + 2 * NKV) * HD), z((NQ + 2 * NKV) * HD), z(NQ * HD), z(NQ * HD)
        self.att8, self.gated = blib.MX8.empty(ROWS, NQ * HD), blib.MX8.empty(ROWS, FF)
        self.delta, self.gu, self.delta2, self.h1, self.h2 = z(D), z(2 * FF), z(D), z(D, torch.float32), z(D, torch.float32)
        self.logits = z(VOCAB, torch.float32)
        f = lambda: torch.zeros(ROWS, dtype=torch.float32, device="cuda")
        self.u, self.temperature, self.top_p, self.top_k, self.token = f(), f(), f(), i32([0] * ROWS), i32([0] * ROWS)
        self.plan = i32([0] * blib.lora_plan_size(ROWS, ADAPTERS))
        self.space = {n: u8(blib.mx8_linear_workspace(x, self.w[n])) for n, x in
                      (("qkv", self.a), ("o", self.att8), ("gu", self.a2), ("down", self.gated), ("head", self.a3))}
        self.lora_space, self.sample_space = u8(blib.lora_workspace(self.ad, ROWS)), u8(blib.sample_workspace(ROWS, VOCAB))
        self.att_space = u8(blib.kv4_attention_workspace(self.cache, NQ, ROWS, B, ROWS, COLS * PAGE))

    def step(self):
        s, heads = self, lambda t: t.unflatten(1, (-1, HD))
        blib.release_pages(s.len, s.done, s.table, s.ring, s.state, PAGE, s.state, s.len)
        blib.plan_pages(s.len, s.new, s.table, s.ring, s.state, PAGE, s.state, s.len, s.cu, s.pos, s.slots, s.refused)
        blib.lora_plan(s.ids, ADAPTERS, s.plan)
        blib.add_rmsnorm(s.h, s.norms[0], y=s.y, mx8=s.a, pos=s.pos)
        blib.mx8_linear(s.a, s.w["qkv"], s.qkv_y, s.space["qkv"])
        blib.lora_add(s.ad, s.y, s.qkv_y, s.qkv, s.plan, s.lora_space)
        q, k, v = heads(s.qkv).split((NQ, NKV, NKV), 1)
        blib.kv4_append_qkv(s.cache, q, k, v, s.pos, s.slots, heads(s.q), q_norm=s.head_norms[0], k_norm=s.head_norms[1])
        blib.kv4_attention(s.cache, heads(s.q), heads(s.att), s.table, s.len, s.cu, ROWS, COLS * PAGE, s.att_space)
        blib.mx8_quantize(s.att, s.att8, pos=s.pos)
        blib.mx8_linear(s.att8, s.w["o"], s.delta, s.space["o"])
        blib.add_rmsnorm(s.h, s.norms[1], delta=s.delta, h_out=s.h1, mx8=s.a2, pos=s.pos)
        blib.mx8_linear(s.a2, s.w["gu"], s.gu, s.space["gu"])
        blib.mx8_quantize(s.gu[:, FF:], s.gated, gate=s.gu[:, :FF], pos=s.pos)
        blib.mx8_linear(s.gated, s.w["down"], s.delta2, s.space["down"])
        blib.add_rmsnorm(s.h1, s.norms[2], delta=s.delta2, h_out=s.h2, mx8=s.a3, pos=s.pos)
        blib.mx8_linear(s.a3, s.w["head"], s.logits, s.space["head"])
        blib.sample(s.logits, s.u, s.token, s.sample_space, s.temperature, top_k=s.top_k, top_p=s.top_p)

    def feed(self, g, news, ended):
        """The step's rows, adapters and sampling parameters; every output cleared to 5."""
        rows = sum(news)
        self.new.copy_(i32(news))
        self.done.copy_(torch.tensor([b in ended for b in range(B)], dtype=torch.uint8))
        self.h.copy_(torch.randn((ROWS, D), generator=g))
        ids = torch.cat([torch.full((n,), int(torch.randint(-1, ADAPTERS, (), generator=g))) for n in news] + [torch.full((ROWS - rows,), -2)])
        self.ids.copy_(ids)
        self.u.copy_(torch.rand(ROWS, generator=g))
        self.temperature.copy_(torch.tensor([0.0, 0.7, 1.0])[torch.randint(0, 3, (ROWS,), generator=g)])
        self.top_p.copy_(torch.tensor([0.5, 0.9, 1.0])[torch.randint(0, 3, (ROWS,), generator=g)])
        self.top_k.copy_(torch.tensor([0, 1, 40])[torch.randint(0, 3, (ROWS,), generator=g)])
        for t in self.outputs():
            t.fill_(5)
        return rows

    def outputs(self):
        eight = [t for m in (self.a, self.a2, self.a3, self.att8, self.gated) for t in m._keep]
        return [self.y, self.qkv_y, self.qkv, self.q, self.att, self.delta, self.gu, self.delta2, self.h1, self.h2, self.logits, self.token, *eight]

    def state_now(self):
        return [self.len, self.table, self.state, self.pos, self.slots, self.plan[:4], *self.cache._keep]


def check_norm(s, h, w, y, m, rows):
    x = h[:rows].cpu().double()
    want = x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6) * w.cpu().double()
    if y is not None:
        err = (y[:rows].cpu().double() - want).abs()
        assert (err <= (22 * U + ROUND[s.dt]) * want.abs()).all() and (y[rows:] == 5).all()
    near_8bit(m.rows(0, rows), want, 22 * U)
    assert (m._keep[0][rows:] == 5).all() and (m._keep[1][rows:] == 5).all()


def check_linear(x, w, out, rows):
    want, tol = linear_tolerance(x.rows(0, rows), w, out.dtype)
    assert ((out[:rows].double() - want).abs() <= tol).all()


STEPS = [([30, 1, 0, 17], []), ([1, 1, 20, 1], []), ([1, 1, 1, 1], []), ([40, 0, 1, 1], [0]), ([0, 0, 0, 0], []), ([1, 1, 1, 1], [1]),
         ([1, 50, 1, 1], []), ([5, 1, 1, 1], [2, 3]), ([1, 0, 0, 0], [])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_of_a_block_eager_and_captured(dtype):
    """Each operator against its reference on what it was given; a captured
    step, replayed with eager work between, leaves the same bits."""
    s, c = Served(DT[dtype]), Served(DT[dtype])
    g, gc = gen(3), gen(3)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.step()
    for news, ended in STEPS:
        rows = s.feed(g, news, ended)
        s.step()
        c.feed(gc, news, ended)
        graph.replay()
        torch.cuda.synchronize()
        assert not s.refused.any()
        # padding leaves a projection's rows free; tokens and plans of live rows
        for name, (x, y) in enumerate(zip(s.outputs(), c.outputs())):
            assert torch.equal(x[:rows], y[:rows]), name
        for x, y in zip(s.state_now(), c.state_now()):
            assert torch.equal(x, y)
        if rows == 0:
            continue
        check_norm(s, s.h, s.norms[0], s.y, s.a, rows)
        check_linear(s.a, s.w["qkv"], s.qkv_y, rows)
        ids = s.ids.tolist()
        want, tol = lora_reference(s.ad, s.y[:rows], s.qkv_y[:rows], ids[:rows])
        assert ((s.qkv[:rows].cpu().double() - want).abs() <= tol).all() and (s.qkv[rows:] == 5).all()
        assert (s.att[:rows] != 5).any() and (s.att[rows:] == 5).all()
        near_8bit(s.att8.rows(0, rows), s.att[:rows].cpu().double(), 0)
        check_linear(s.att8, s.w["o"], s.delta, rows)
        assert torch.equal(s.h1[:rows], s.h[:rows] + s.delta[:rows].float()) and (s.h1[rows:] == 5).all()
        check_norm(s, s.h1, s.norms[1], None, s.a2, rows)
        check_linear(s.a2, s.w["gu"], s.gu, rows)
        gate, up = s.gu[:rows, :FF].cpu().double(), s.gu[:rows, FF:].cpu().double()
        near_8bit(s.gated.rows(0, rows), gate / (1 + torch.exp(-gate)) * up, 8 * U)
        check_linear(s.gated, s.w["down"], s.delta2, rows)
        assert torch.equal(s.h2[:rows], s.h1[:rows] + s.delta2[:rows].float()) and (s.h2[rows:] == 5).all()
        check_norm(s, s.h2, s.norms[2], None, s.a3, rows)
        check_linear(s.a3, s.w["head"], s.logits, rows)
        logits = s.logits.cpu()
        for r in range(rows):
            want = token_of(logits[r], s.u[r].item(), s.temperature[r].item(), s.top_k[r].item(), s.top_p[r].item(), 0.0)
            assert s.token[r].item() == want


def calls(dtype, rows=70):
    """One call of each operator with buffers and workspaces of its own:
    (enqueue(stream), outputs)."""
    g, dt = gen(rows), DT[dtype]
    x, w = linear_case(rows, 528, 1280, rows)
    wide = torch.randn((rows, 1280), generator=g).cuda()
    delta = torch.randn((rows, 1280), generator=g).to(dt).cuda()
    weight = torch.rand(1280, generator=g).to(dt).cuda()
    ad = adapters_of(5, 32, 1280, 528, dt, 1)
    ids = i32(torch.randint(-1, 5, (rows,), generator=g).tolist())
    logits = (4 * torch.randn((rows, 9001), generator=g)).to(dt).cuda()
    u = torch.rand(rows, generator=g).cuda()
    t, p = torch.full_like(u, 0.8), torch.full_like(u, 0.95)
    u8 = lambda n: torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    o = dict(h=torch.zeros_like(wide), y=torch.zeros_like(delta), lin=torch.zeros((rows, 528), dtype=dt, device="cuda"),
             lora=torch.zeros((rows, 528), dtype=dt, device="cuda"), read=torch.zeros((rows, 1280), dtype=dt, device="cuda"), token=i32([0] * rows))
    m, m2 = blib.MX8.empty(rows, 1280), blib.MX8.empty(rows, 1280)
    plan = i32([0] * blib.lora_plan_size(rows, 5))
    ws, ls, ss = u8(blib.mx8_linear_workspace(x, w)), u8(blib.lora_workspace(ad, rows)), u8(blib.sample_workspace(rows, 9001))

    def enqueue(stream=None):
        blib.add_rmsnorm(wide, weight, delta=delta, h_out=o["h"], y=o["y"], mx8=m, stream=stream)
        blib.mx8_quantize(o["y"], m2, gate=delta, stream=stream)
        blib.mx8_read(m2, o["read"], stream=stream)
        blib.mx8_linear(m, w, o["lin"], ws, stream=stream)
        blib.lora_plan(ids, 5, plan, stream=stream)
        blib.lora_add(ad, o["y"], o["lin"], o["lora"], plan, ls, stream=stream)
        blib.sample(logits, u, o["token"], ss, t, top_p=p, stream=stream)
    return enqueue, [*o.values(), *m._keep, *m2._keep]


def cleared(outputs):
    for t in outputs:
        t.zero_()


@pytest.mark.parametrize("rows", [1, 70, 600])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_given_streams_and_graphs_at_once(dtype, rows):
    first, second = calls(dtype, rows), calls(dtype, rows)
    first[0]()
    torch.cuda.synchronize()
    want = [t.clone() for t in first[1]]
    assert all(t.any() for t in want[:5])
    same = lambda outputs: all(torch.equal(a, b) for a, b in zip(outputs, want))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    # two streams, given to the calls, their work interleaved
    for _, outputs in (first, second):
        cleared(outputs)
    torch.cuda.synchronize()
    for _ in range(3):
        for s, (enqueue, _) in zip(streams, (first, second)):
            enqueue(s)
    torch.cuda.synchronize()
    assert same(first[1]) and same(second[1])
    # two graphs, each with its own buffers, replayed side by side
    graphs = []
    for enqueue, _ in (first, second):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            enqueue(torch.cuda.current_stream())
        graphs.append(graph)
    for _ in range(4):
        for _, outputs in (first, second):
            cleared(outputs)
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert same(first[1]) and same(second[1])
        first[0]()                                             # eager work between the replays
        torch.cuda.synchronize()
        assert same(first[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_workspace_of_more_rows_serves_fewer(dtype):
    u8 = lambda n: torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    most, w = linear_case(700, 260, 4224, 1)
    ad = adapters_of(3, 24, 264, 136, DT[dtype], 2)
    ws, ls, ss = u8(blib.mx8_linear_workspace(most, w)), u8(blib.lora_workspace(ad, 1100)), u8(blib.sample_workspace(64, 700))
    for rows in (700, 1, 40, 300, 16, 128):
        x = most.rows(0, rows)
        out = torch.empty((rows, 260), dtype=DT[dtype], device="cuda")
        blib.mx8_linear(x, w, out, ws)
        assert torch.equal(out, run_linear(x, w, DT[dtype]))
    for rows in (1100, 3, 300):
        v, y = torch.randn((rows, 264), generator=gen(rows)).to(DT[dtype]).cuda(), torch.zeros((rows, 136), dtype=DT[dtype], device="cuda")
        ids, out = [r % 4 - 1 for r in range(rows)], torch.empty_like(y)
        plan = i32([0] * blib.lora_plan_size(1100, 3))
        blib.lora_plan(i32(ids), 3, plan)
        blib.lora_add(ad, v, y, out, plan, ls)
        assert torch.equal(out, run_lora(ad, v, y, torch.empty_like(y), ids))
    for rows in (64, 1, 7):
        l = torch.randn((rows, 700), generator=gen(rows)).to(DT[dtype]).cuda()
        token, f = i32([0] * rows), torch.full((rows,), 0.6, device="cuda")
        blib.sample(l, f, token, ss, f)
        assert token.tolist() == [token_of(r, f[0].item(), f[0].item(), 0, 1.0, 0.0) for r in l.cpu()]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_apart(dtype):
    """Rows a gigabyte apart: offsets past 32 bits, and code rows further
    apart than the projection's tiles reach."""
    dt, rows, k, n, far = DT[dtype], 6, 272, 136, 2 ** 30 + 4096
    def apart(width, t, at):
        one = torch.empty((), dtype=t).element_size()
        buf = torch.empty(rows * far, dtype=torch.uint8, device="cuda")[at * one:]
        return buf[:buf.numel() // one * one].view(t).as_strided((rows, width), (far // one, 1))
    eight = lambda m, at: blib.MX8(apart(m.shape[1], torch.uint8, at).copy_(m._keep[0]), apart(16, torch.uint8, at).copy_(m._keep[1]))
    x, w = linear_case(rows, n, k, 3)
    w6 = linear_case(rows, rows, k, 4)[1]
    xf = eight(x, 64)
    out = apart(n, dt, 3)
    run_linear(xf, w, dt, out)
    assert torch.equal(out, run_linear(x, w, dt))
    assert torch.equal(run_linear(x, eight(w6, 16), dt), run_linear(x, w6, dt))
    del out
    # norm, 8-bit rows and back
    h, delta = torch.randn((rows, k), generator=gen(1)).cuda(), torch.randn((rows, k), generator=gen(2)).to(dt).cuda()
    weight = torch.rand(k, generator=gen(3)).to(dt).cuda()
    y, m, h_out = torch.empty_like(delta), blib.MX8.empty(rows, k), torch.empty_like(h)
    blib.add_rmsnorm(h, weight, delta=delta, h_out=h_out, y=y, mx8=m)
    hf, yf, df = apart(k, torch.float32, 32).copy_(h), apart(k, dt, 16), apart(k, dt, 16).copy_(delta)
    blib.add_rmsnorm(hf, weight, delta=df, y=yf, mx8=xf)
    assert torch.equal(hf, h_out) and torch.equal(yf, y) and torch.equal(xf._keep[0], m._keep[0])
    assert torch.equal(xf._keep[1][:, :9], m._keep[1][:, :9])
    blib.mx8_quantize(df, xf, gate=yf)
    blib.mx8_quantize(delta, m, gate=y)
    assert torch.equal(xf._keep[0], m._keep[0])
    blib.mx8_read(xf, yf)
    blib.mx8_read(m, y)
    assert torch.equal(yf, y)
    # adapters, in place
    ad, ids = adapters_of(2, 8, k, n, dt, 1), [0, 1, -1, 0, 1, 0]
    v = torch.randn((rows, n), generator=gen(5)).to(dt).cuda()
    vf = apart(n, dt, 64).copy_(v)
    df.copy_(delta)
    run_lora(ad, df, vf, vf, ids)
    assert torch.equal(vf, run_lora(ad, delta, v, torch.empty_like(v), ids))
    # logits
    l = torch.randn((rows, 5003), generator=gen(6)).to(dt).cuda()
    lf = apart(5003, dt, 1).copy_(l)
    u, t = torch.rand(rows, generator=gen(7)).cuda(), torch.ones(rows, device="cuda")
    token, ws = i32([0] * rows), torch.empty(blib.sample_workspace(rows, 5003), dtype=torch.uint8, device="cuda")
    blib.sample(lf, u, token, ws, t)
    assert token.tolist() == [token_of(l.cpu()[i], u[i].item(), 1.0, 0, 1.0, 0.0) for i in range(rows)]


def test_more_rows_than_workgroups():
    """Rows past the largest grids, which then take several each."""
    n = 2 ** 20 + 77
    h, w = torch.randn((n, 16), device="cuda"), torch.rand(16, device="cuda")
    y, m = torch.empty_like(h), blib.MX8.empty(n, 16)
    blib.add_rmsnorm(h, w, y=y, mx8=m)
    part, few = torch.empty((100, 16), device="cuda"), blib.MX8.empty(100, 16)
    for at in (0, 2 ** 20 - 50, n - 100):
        blib.add_rmsnorm(h[at:at + 100], w, y=part, mx8=few)
        assert torch.equal(y[at:at + 100], part) and torch.equal(m._keep[0][at:at + 100], few._keep[0])
    n, width = 2 ** 24, 144                                   # 2^28 lanes in a grid
    x = torch.randint(-30000, 30000, (n, width), dtype=torch.int16, device="cuda").view(torch.bfloat16).nan_to_num_(1.0, 1.0, 1.0)
    m, few = blib.MX8.empty(n, width), blib.MX8.empty(1000, width)
    blib.mx8_quantize(x, m)
    out, part = torch.empty_like(x), torch.empty((1000, width), dtype=x.dtype, device="cuda")
    blib.mx8_read(m, out)
    for at in (0, n * 3 // 4, n - 1000):
        blib.mx8_quantize(x[at:at + 1000], few)
        blib.mx8_read(few, part)
        assert torch.equal(m._keep[0][at:at + 1000], few._keep[0]) and torch.equal(m._keep[1][at:at + 1000], few._keep[1])
        assert torch.equal(out[at:at + 1000], part)


def test_a_single_row_of_rows_apart():
    """A row's own width of scale bytes may be odd."""
    codes, scales = torch.zeros((3, 80), dtype=torch.uint8, device="cuda"), torch.zeros((3, 32), dtype=torch.uint8, device="cuda")
    x = torch.randn((3, 64), generator=gen(1)).cuda()
    m = blib.MX8(codes[:, :64], scales[:, :20])
    blib.mx8_quantize(x, m)
    assert torch.equal(values(m), values(mx8_of(x)))
    one = m.rows(1, 2)
    blib.mx8_quantize(x[2:], one)
    assert torch.equal(values(m)[1], values(m)[2])


def test_no_rows():
    z = lambda *s: torch.zeros(s, device="cuda")
    m, w = blib.MX8.empty(0, 48), blib.MX8.empty(8, 48)
    blib.add_rmsnorm(z(0, 48), z(48), delta=z(0, 48), y=z(0, 48), mx8=m)
    blib.mx8_quantize(z(0, 48), m)
    blib.mx8_read(m, z(0, 48))
    ws = torch.zeros(blib.mx8_linear_workspace(m, w), dtype=torch.uint8, device="cuda")
    blib.mx8_linear(m, w, z(0, 8), ws)
    ad = blib.Adapters(z(2, 8, 48), z(2, 8, 8), z(2))
    plan = i32([7] * 8)
    blib.lora_plan(i32([]), 2, plan)
    blib.lora_add(ad, z(0, 48), z(0, 8), z(0, 8), plan, ws)
    blib.sample(z(0, 9), z(0), i32([]), ws, z(0))
    torch.cuda.synchronize()
    assert (plan == 7).all()


def test_refusals():
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device="cuda")
    m, w = blib.MX8.empty(3, 48), blib.MX8.empty(8, 48)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError, match="different shapes"):
        blib.MX8(z(3, 528, t=torch.uint8), z(3, 16, t=torch.uint8))
    with pytest.raises(ValueError, match="contiguous"):
        blib.MX8(z(48, 3, t=torch.uint8).T, z(3, 16, t=torch.uint8))
    with pytest.raises(ValueError, match="mx8: expected shape"):
        blib.add_rmsnorm(z(4, 48), z(48), mx8=m)
    with pytest.raises(ValueError, match="weight: expected at least 48"):
        blib.add_rmsnorm(z(3, 48), z(40), mx8=m)
    with pytest.raises(TypeError, match="delta: expected float32"):
        blib.add_rmsnorm(z(3, 48), z(48), delta=z(3, 48, t=torch.bfloat16), mx8=m)
    with pytest.raises(ValueError, match="h_out: expected shape"):
        blib.add_rmsnorm(z(3, 48), z(48), delta=z(3, 48), h_out=z(2, 48), mx8=m)
    with pytest.raises(ValueError, match="pos: expected at least 3"):
        blib.add_rmsnorm(z(3, 48), z(48), mx8=m, pos=i32([0]))
    for args in ((z(3, 40), z(40)), (z(3, 64)[:, 1:49], z(48)), (z(3, 50)[:, :48], z(48)), (z(3, 48), z(52)[2:])):
        with pytest.raises(blib.BuddyError):
            blib.add_rmsnorm(*args, y=z(3, args[0].shape[1]))
    with pytest.raises(blib.BuddyError):
        blib.add_rmsnorm(z(3, 48), z(48))                      # nothing to write
    with pytest.raises(blib.BuddyError):
        blib.add_rmsnorm(z(1, 48).expand(3, 48), z(48), mx8=m)   # rows of one place
    with pytest.raises(ValueError, match="x: expected shape"):
        blib.mx8_quantize(z(3, 64), m)
    with pytest.raises(TypeError, match="gate: expected float32"):
        blib.mx8_quantize(z(3, 48), m, gate=z(3, 48, t=torch.bfloat16))
    with pytest.raises(TypeError, match="out: expected float32 or bfloat16"):
        blib.mx8_read(m, z(3, 48, t=torch.float16))
    with pytest.raises(ValueError, match="out: expected shape"):
        blib.mx8_linear(m, w, z(3, 9), ws)
    with pytest.raises(blib.BuddyError):
        blib.mx8_linear(m, w, z(3, 8), ws[:8])
    with pytest.raises(blib.BuddyError):
        blib.mx8_linear(m, w, z(3, 8), ws[8:])
    with pytest.raises(blib.BuddyError):
        blib.mx8_linear(m, blib.MX8.empty(8, 64), z(3, 8), ws)
    ad = blib.Adapters(z(2, 8, 48), z(2, 24, 8), z(2))
    plan = i32([0] * blib.lora_plan_size(3, 2))
    with pytest.raises(ValueError, match="plan: expected at least"):
        blib.lora_plan(i32([0, 1, 0]), 2, plan[:9])
    with pytest.raises(ValueError, match="plan: expected at least"):
        blib.lora_add(ad, z(3, 48), z(3, 24), z(3, 24), plan[:9], ws)
    with pytest.raises(TypeError, match="x: expected float32"):
        blib.lora_add(ad, z(3, 48, t=torch.bfloat16), z(3, 24), z(3, 24), plan, ws)
    with pytest.raises(ValueError, match="y: expected shape"):
        blib.lora_add(ad, z(3, 48), z(3, 32), z(3, 24), plan, ws)
    with pytest.raises(blib.BuddyError):
        blib.lora_add(ad, z(3, 48), z(3, 24), z(3, 24), plan, ws[:16])
    with pytest.raises(blib.BuddyError):
        blib.lora_plan(i32([0]), 5000, plan)
    with pytest.raises(ValueError, match="token: expected at least 3"):
        blib.sample(z(3, 9), z(3), i32([0]), ws, z(3))
    with pytest.raises(TypeError, match="temperature: expected float32"):
        blib.sample(z(3, 9), z(3), i32([0] * 3), ws, z(3, t=torch.bfloat16))
    with pytest.raises(blib.BuddyError):
        blib.sample(z(3, 9), z(3), i32([0] * 3), ws[:64], z(3))
    with pytest.raises(ValueError, match="contiguous"):
        blib.sample(z(9, 3).T, z(3), i32([0] * 3), ws, z(3))
