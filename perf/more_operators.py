"""Measured calls of the operators that surround attention in a served block and end its
step: residual and norm with 8-bit rows, 8-bit rows of activations, projections of them,
low-rank adapters of many requests, sampling.

listed() names the cases, draw() gives more of the same ranges, prepare() makes what a
program holds before the call, run() is one pass (the plain form, or the library's calls
where `own` is set), work() what a pass cannot do without, exact() its answer in 64 bits.

8-bit rows: e4m3 codes [rows][width]; 32 neighbours of a row share a power-of-two scale
(E8M0) in [rows][16 for each 512 of the width], the last group of a row may be short.  A
group's exponent is the least e with amax <= 448 * 2^e, kept within -117..120.
"""
import math

import torch

own = False

# d_model, query heads, KV heads, head_dim, d_ffn of the model shapes that the library's benchmarks use
SHAPES = {"tiny": (256, 4, 2, 64, 688), "llama3_8b": (4096, 32, 8, 128, 14336), "qwen2_7b": (3584, 28, 4, 128, 18944), "mha_13b": (5120, 40, 40, 128, 13824)}
EPS = 1e-6
UNIT = 2.0**40  # a token's weight counts in units of 2^-40 of the likeliest token's


def _case(name, op, **kw):
    c = dict(name=name, op=op, **kw)
    if not name:
        del c["name"]
    return c


def listed():
    return [
        # the residual's addition and norm before a projection, one token of one conversation
        _case("norm_one", "norm", shape="llama3_8b", rows=1, hidden="f32", dtype="bf16", out="mx8", delta=True, pad=False),
        # the same for prompts admitted together, a few rows of padding behind them
        _case("norm_prompt", "norm", shape="mha_13b", rows=8192, hidden="f32", dtype="bf16", out="mx8", delta=True, pad=True),
        # the gated activation of a decode batch, made ready for the down projection
        _case("act_batch", "quant", shape="qwen2_7b", rows=64, gate=True, dtype="bf16", pad=False),
        # a prompt's attention outputs, made ready for the output projection
        _case("rows_prompt", "quant", shape="llama3_8b", rows=8195, gate=False, dtype="bf16", pad=False),
        # one token through the fused query, key and value projection
        _case("linear_one", "linear", shape="llama3_8b", proj="qkv", rows=1, dtype="bf16"),
        # the batched serving workload of the multi-head model through gate and up
        _case("linear_batch", "linear", shape="mha_13b", proj="gate_up", rows=96, dtype="bf16"),
        # prompts through gate and up
        _case("linear_prompt", "linear", shape="llama3_8b", proj="gate_up", rows=8192, dtype="bf16"),
        # one token, one adapter
        _case("lora_one", "lora", shape="llama3_8b", proj="qkv", rows=1, rank=16, adapters=8, mixed=True, none=0.0, dtype="bf16"),
        # a decode batch in which nearly every request has an adapter of its own
        _case("lora_batch", "lora", shape="mha_13b", proj="o", rows=96, rank=32, adapters=48, mixed=True, none=0.2, dtype="bf16"),
        # prompts of a few adapters admitted together
        _case("lora_prompt", "lora", shape="qwen2_7b", proj="gate_up", rows=4099, rank=64, adapters=5, mixed=False, none=0.2, dtype="bf16"),
        # the next token of one conversation
        _case("sample_one", "sample", batch=1, vocab=128000, dtype="f32", kind="mixed"),
        # of a large batch, each request with settings of its own, an odd vocabulary
        _case("sample_batch", "sample", batch=256, vocab=151001, dtype="f32", kind="mixed"),
    ]


def _io(shape, proj):
    d, nq, nkv, hd, f = SHAPES[shape]
    return {"qkv": (d, (nq + 2 * nkv) * hd), "o": (nq * hd, d), "gate_up": (d, 2 * f), "down": (f, d), "head": (d, 128000 if d > 256 else 1003)}[proj]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["norm", "norm", "quant", "linear", "linear", "linear", "lora", "lora", "lora", "sample", "sample"])
    if op == "sample":
        dtype = rng.choice(["f32", "f32", "bf16"])
        return _case("", op, batch=log_int(1, 256), vocab=log_int(1000, 151001), dtype=dtype, kind=rng.choice(["mixed", "mixed", "mixed", "plain", "greedy", "flat"]))
    shape = rng.choice(["llama3_8b", "llama3_8b", "qwen2_7b", "mha_13b", "tiny"])
    d, f = SHAPES[shape][0], SHAPES[shape][4]
    if op == "norm":
        hidden, dtype = rng.choice([("f32", "bf16"), ("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
        return _case("", op, shape=shape, rows=log_int(1, min(16384, 8192 * 5120 // d)) // (2 if dtype == "f32" else 1) + 1, hidden=hidden, dtype=dtype,
                     out=rng.choice(["mx8", "mx8", "y", "both"]), delta=rng.random() < 0.85, pad=rng.random() < 0.3)
    if op == "quant":
        gate, dtype = rng.random() < 0.6, rng.choice(["bf16", "bf16", "bf16", "f32"])
        most = 8195 * 4096 // ((3 * f if gate else d) * (2 if dtype == "f32" else 1))
        return _case("", op, shape=shape, rows=log_int(1, min(16384, most)), gate=gate, dtype=dtype, pad=rng.random() < 0.3)
    if op == "linear":
        proj = rng.choice(["qkv", "o", "gate_up", "down", "head"])
        k, n = _io(shape, proj)
        rows = log_int(1, 16 if rng.random() < 0.3 else min(8192, 8192 * 4096 * 28672 // (k * n)))
        if proj == "head":  # the last token of each sequence
            rows = min(rows, 256)
        return _case("", op, shape=shape, proj=proj, rows=rows, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    proj = rng.choice(["qkv", "o", "gate_up", "down"])
    k, n = _io(shape, proj)
    mixed, rank = rng.random() < 0.6, rng.choice([8, 16, 16, 32, 64, 128])
    dtype = "f32" if rng.random() < (0.6 if shape == "tiny" else 0.1) else "bf16"
    rows = log_int(1, 256) if mixed else log_int(2, min(4096, 4099 * 64 * 37888 // (n * rank)))
    if dtype == "f32":
        rows = (rows + 7) // 8
    return _case("", op, shape=shape, proj=proj, rows=rows, rank=rank, adapters=log_int(1, 48 if mixed else 6), mixed=mixed, none=rng.choice([0.0, 0.2, 0.5]),
                 dtype=dtype)


# ------------------------------------------------------------------ inputs


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _room(width):
    """Bytes of a row's scales."""
    return (width + 511) // 512 * 16


def _positions(case):
    """Rows that a step runs; the others are padding behind them."""
    return case["rows"] - (case["rows"] // 9 if case["pad"] else 0)


def _row_adapters(case, host):
    n, have = case["rows"], case["adapters"]
    if case["mixed"]:  # single tokens of requests in any order
        ids = torch.randint(0, have, (n,), generator=host)
        return torch.where(torch.rand(n, generator=host) < case["none"], -1, ids)
    # prompts one behind another, of uneven lengths
    parts = 2 * have + 1
    ends = torch.sort(torch.randint(0, n + 1, (parts - 1,), generator=host)).values
    of = torch.randint(0, have, (parts,), generator=host)
    of = torch.where(torch.rand(parts, generator=host) < case["none"], -1, of)
    return of[torch.searchsorted(ends, torch.arange(n), right=True)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    zeros = lambda *s, dtype=torch.uint8: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    st = dict(case=case)
    if case["op"] == "sample":
        b, v = case["batch"], case["vocab"]
        # a spread of unlikely tokens and a few likely ones, some ruled out by a grammar
        x = (0.5 if case["kind"] == "flat" else 2.2) * randn(b, v)
        x[torch.arange(b, device="cuda")[:, None], torch.randint(0, v, (b, 12), device="cuda", generator=gen)] += 6 + 3 * randn(b, 12)
        x[:, :: 97] = -math.inf
        rows = torch.randint(0, 4, (4, b), generator=host)
        pick = lambda i, values, dt: torch.tensor(values, dtype=dt)[rows[i]].cuda()  # noqa: E731
        if case["kind"] == "mixed":
            st.update(temperature=pick(0, [0.0, 0.6, 1.0, 1.3], torch.float32), top_k=pick(1, [0, 1, 40, 1000], torch.int32),
                      top_p=pick(2, [0.5, 0.9, 0.95, 1.0], torch.float32), min_p=pick(3, [0.0, 0.0, 0.02, 0.1], torch.float32))
            if b == 1:
                st["temperature"].fill_(0.8), st["top_k"].fill_(0), st["top_p"].fill_(0.95), st["min_p"].fill_(0.0)
        else:
            one = lambda value, dt: torch.full((b,), value, dtype=dt, device="cuda")  # noqa: E731
            st.update(temperature=one(0.0 if case["kind"] == "greedy" else 1.0, torch.float32), top_k=one(0, torch.int32),
                      top_p=one(0.9 if case["kind"] == "flat" else 1.0, torch.float32), min_p=one(0.0, torch.float32))
        st.update(logits=x.to(_dtype(case["dtype"])), u=torch.rand(b, device="cuda", generator=gen), tokens=zeros(b, dtype=torch.int32), workspace=None)
        return st
    dt, rows = _dtype(case["dtype"]), case["rows"]
    if case["op"] in ("norm", "quant"):
        pos = torch.arange(rows, dtype=torch.int32)
        pos[_positions(case) :] = -1
        st.update(pos=pos.cuda() if case["pad"] else None)
    if case["op"] == "norm":
        d = SHAPES[case["shape"]][0]
        hidden = _dtype(case["hidden"])
        # residual streams have a few large channels
        big = 1 + 20 * (torch.rand(d, device="cuda", generator=gen) < 0.01)
        st.update(h=(3 * randn(rows, d) * big).to(hidden), h_out=zeros(rows, d, dtype=hidden), delta=randn(rows, d).to(dt) if case["delta"] else None,
                  w=(1 + 0.2 * randn(d)).to(dt), codes=zeros(rows, d), scales=zeros(rows, _room(d)), y=zeros(rows, d, dtype=dt),
                  values=zeros(rows, d, dtype=torch.bfloat16))
    elif case["op"] == "quant":
        d, f = SHAPES[case["shape"]][0], SHAPES[case["shape"]][4]
        width = f if case["gate"] else d
        x = randn(rows, 2 * f if case["gate"] else d).to(dt)  # gate and up side by side, as the projection leaves them
        st.update(x=x[:, -width:], gate=x[:, :f] if case["gate"] else None, codes=zeros(rows, width), scales=zeros(rows, _room(width)),
                  values=zeros(rows, width, dtype=torch.bfloat16))
    elif case["op"] == "linear":
        k, n = _io(case["shape"], case["proj"])
        x, w = _mx8(randn(rows, k)), _mx8(randn(n, k) / math.sqrt(k))
        st.update(x_codes=x[0], x_scales=x[1], w_codes=w[0], w_scales=w[1], out=zeros(rows, n, dtype=dt), workspace=None)
    else:
        k, n = _io(case["shape"], case["proj"])
        r, have = case["rank"], case["adapters"]
        st.update(x=randn(rows, k).to(dt), a=(randn(have, r, k) / math.sqrt(k)).to(dt), b=(0.3 * randn(have, n, r)).to(dt),
                  scale=0.25 + torch.rand(have, device="cuda", generator=gen), ids=_row_adapters(case, host).to(torch.int32).cuda(), y=randn(rows, n).to(dt),
                  out=zeros(rows, n, dtype=dt), plan=None)
    return st


# ------------------------------------------------------------- plain forms


def _pow2(e):
    """2^e of whole numbers -126..127, fp32, exact (pow is not for every e)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _groups(x):
    """[rows][width] -> [rows][groups][32], the last group filled up with zeros."""
    return torch.nn.functional.pad(x, (0, -x.shape[1] % 32)).unflatten(1, (-1, 32))


def _mx8(x):
    """fp32 [rows][width] -> codes [rows][width], scales [rows][room]."""
    rows, width = x.shape
    g = _groups(x)
    amax = g.abs().amax(-1)
    m, e = torch.frexp(amax)  # 448 = 0.875 * 2^9
    e = torch.where(amax > 0, e - 9 + (m > 0.875).int(), -117).clamp(-117, 120)
    codes = (g * _pow2(-e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    scales = torch.full((rows, _room(width)), 127, dtype=torch.uint8, device=x.device)
    scales[:, : e.shape[1]] = (e + 127).to(torch.uint8)
    return codes.flatten(1)[:, :width].contiguous(), scales


def _values(codes, scales):
    """fp32 values of 8-bit rows."""
    g = _groups(codes).view(torch.float8_e4m3fn).float()
    s = scales[:, : g.shape[1]].int() - 127
    return (g * torch.where(s < -126, 2.0**-127, _pow2(s))[..., None]).flatten(1)[:, : codes.shape[1]]


def _live(st, *outputs):
    """Outputs of the rows that are no padding; the rest stay as the buffers are, zero."""
    if st["pos"] is None:
        return list(outputs)
    return [torch.where((st["pos"] >= 0)[:, None], x, torch.zeros((), dtype=x.dtype, device=x.device)) for x in outputs]


def _plain_sample(st):
    x = st["logits"].double()
    x = torch.where(x.isnan(), -math.inf, x)
    b, v = x.shape
    top = x.amax(1, keepdim=True)
    t = st["temperature"].double()[:, None]
    greedy = ~(t > 0)
    z = torch.where(x == top, 0.0, (x - top) / torch.where(greedy, 1.0, t))
    weight = torch.round(torch.exp(z) * UNIT).long()
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    w = weight.gather(1, order)
    at = torch.arange(v, device="cuda")
    # the most likely tokens, then those near enough to the likeliest
    k = st["top_k"].long()[:, None]
    k = torch.where((k <= 0) | (k > v), v, k)
    w = torch.where((at < k) & (w >= (st["min_p"].double()[:, None] * UNIT).clamp(max=UNIT)), w, 0)
    # of those the fewest that hold a share top_p of the weight
    need = torch.ceil(st["top_p"].double()[:, None].clamp(max=1.0) * w.sum(1, keepdim=True).double()).long()
    sums = w.cumsum(1)
    w = torch.where((sums - w < need) | (at == 0), w, 0)
    # the one at u of the rest, in the order of the vocabulary
    kept = torch.zeros_like(weight).scatter_(1, order, w)
    total = kept.sum(1, keepdim=True)
    target = torch.floor(st["u"].double()[:, None] * total.double()).long()
    target = torch.minimum(target, total - 1)
    token = (kept.cumsum(1) <= target).sum(1)
    token = torch.where(greedy[:, 0], order[:, 0], token)
    return torch.where(top[:, 0] == -math.inf, -1, token).int()


def run(st):
    op = st["case"]["op"]
    if own:
        return _own(st, op)
    if op == "norm":
        h = st["h"].float()
        if st["delta"] is not None:
            h = (h + st["delta"].float()).to(st["h"].dtype).float()
        y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * st["w"].float()
        outs = [h.to(st["h"].dtype)] if st["delta"] is not None else []
        if st["case"]["out"] != "mx8":
            outs.append(y.to(st["w"].dtype))
        if st["case"]["out"] != "y":
            outs.append(_values(*_mx8(y)).bfloat16())
        return _live(st, *outs)
    if op == "quant":
        x = st["x"].float()
        if st["gate"] is not None:
            g = st["gate"].float()
            x = g / (1 + torch.exp(-g)) * x
        return _live(st, _values(*_mx8(x)).bfloat16())
    if op == "linear":
        return torch.matmul(_values(st["x_codes"], st["x_scales"]), _values(st["w_codes"], st["w_scales"]).T).to(st["out"].dtype)
    if op == "lora":
        # all adapters on all rows, of which a row keeps its own
        have, r, k = st["a"].shape
        t = torch.matmul(st["x"].float(), st["a"].float().view(have * r, k).T).view(-1, have, r)
        mine = st["ids"][:, None] == torch.arange(have, device="cuda")
        t = torch.where(mine[..., None], t * st["scale"][:, None], 0.0)
        add = torch.matmul(t.flatten(1), st["b"].float().permute(0, 2, 1).reshape(have * r, -1))
        return (st["y"].float() + add).to(st["y"].dtype)
    return _plain_sample(st)


def _own(st, op):
    from paper_2606_09514_amd import lib

    if op == "norm":
        out, delta = st["case"]["out"], st["delta"]
        if "mx8" not in st:
            st["mx8"] = lib.MX8(st["codes"], st["scales"])
        lib.add_rmsnorm(st["h"], st["w"], delta=delta, h_out=None if delta is None else st["h_out"], y=None if out == "mx8" else st["y"],
                        mx8=None if out == "y" else st["mx8"], pos=st["pos"], eps=EPS)
        outs = [] if delta is None else [st["h_out"]]
        if out != "mx8":
            outs.append(st["y"])
        if out != "y":
            lib.mx8_read(st["mx8"], st["values"])
            outs.append(st["values"])
        return outs
    if op == "quant":
        if "mx8" not in st:
            st["mx8"] = lib.MX8(st["codes"], st["scales"])
        lib.mx8_quantize(st["x"], st["mx8"], gate=st["gate"], pos=st["pos"])
        lib.mx8_read(st["mx8"], st["values"])
        return [st["values"]]
    if op == "linear":
        if st["workspace"] is None:  # kept by a program beside its other buffers
            st["x"], st["w"] = lib.MX8(st["x_codes"], st["x_scales"]), lib.MX8(st["w_codes"], st["w_scales"])
            st["workspace"] = torch.empty(lib.mx8_linear_workspace(st["x"], st["w"]), dtype=torch.uint8, device="cuda")
        lib.mx8_linear(st["x"], st["w"], st["out"], st["workspace"])
        return st["out"]
    if op == "lora":
        if st["plan"] is None:
            rows, have = st["x"].shape[0], st["a"].shape[0]
            st["adapters"] = lib.Adapters(st["a"], st["b"], st["scale"])
            st["plan"] = torch.empty(lib.lora_plan_size(rows, have), dtype=torch.int32, device="cuda")
            st["workspace"] = torch.empty(lib.lora_workspace(st["adapters"], rows), dtype=torch.uint8, device="cuda")
        lib.lora_plan(st["ids"], st["a"].shape[0], st["plan"])
        lib.lora_add(st["adapters"], st["x"], st["y"], st["out"], st["plan"], st["workspace"])
        return st["out"]
    if st["workspace"] is None:
        st["workspace"] = torch.empty(lib.sample_workspace(*st["logits"].shape), dtype=torch.uint8, device="cuda")
    lib.sample(st["logits"], st["u"], st["tokens"], st["workspace"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"])
    return st["tokens"]


# ------------------------------------------------------------------- work


def work(case):
    if case["op"] == "sample":
        size = 4 if case["dtype"] == "f32" else 2
        return dict(bytes=case["batch"] * (case["vocab"] * size + 24), flops=0)
    size, rows = 4 if case["dtype"] == "f32" else 2, case["rows"]
    held = lambda width: width + (width + 31) // 32  # noqa: E731
    if case["op"] == "norm":
        d, live = SHAPES[case["shape"]][0], _positions(case)
        b = (4 if case["hidden"] == "f32" else 2) * (2 if case["delta"] else 1) + (size if case["delta"] else 0)
        b = live * d * (b + (size if case["out"] != "mx8" else 0))
        if case["out"] != "y":  # written, and read back as 16-bit values
            b += (live + rows) * held(d) + 2 * rows * d
        return dict(bytes=b + d * size, flops=5 * live * d)
    if case["op"] == "quant":
        width, live = SHAPES[case["shape"]][4 if case["gate"] else 0], _positions(case)
        return dict(bytes=live * width * size * (2 if case["gate"] else 1) + (live + rows) * held(width) + 2 * rows * width, flops=6 * live * width)
    k, n = _io(case["shape"], case["proj"])
    if case["op"] == "linear":
        return dict(bytes=(rows + n) * held(k) + rows * n * size, flops=2 * rows * k * n)
    ids = _row_adapters(case, torch.Generator().manual_seed(1))
    used, live = len(set(ids.tolist()) - {-1}), int((ids >= 0).sum())
    r = case["rank"]
    return dict(bytes=size * (used * r * (k + n) + live * k + 2 * rows * n) + 4 * rows, flops=2 * live * r * (k + n))


# ------------------------------------------------------------- 64-bit answer


def _pow2_64(e):
    """2^e of whole numbers, 64 bits, exact."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _values64(codes, scales):
    """64-bit values of 8-bit rows, from the bits of the format."""
    c = codes.long()
    e, m = (c >> 3) & 15, (c & 7).double()
    x = torch.where(e > 0, (8 + m) * _pow2_64(e - 10), m * 2.0**-9)
    x = torch.where((c & 127) == 127, math.nan, torch.where(c >= 128, -x, x))
    return x * _pow2_64(scales.long() - 127).repeat_interleave(32, dim=1)[:, : codes.shape[1]]


def _round64(x):
    """Values [rows][width] as 8-bit rows hold them."""
    width = x.shape[1]
    x = _groups(x.double())
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(amax.clamp(min=1e-300) / 448))
    e = torch.where(amax > 448 * _pow2_64(e), e + 1, torch.where(amax <= 448 * _pow2_64(e - 1), e - 1, e)).clamp(-117, 120)
    a = x / _pow2_64(e)
    step = _pow2_64(torch.floor(torch.log2(a.abs().clamp(min=2.0**-6))) - 3)
    return (torch.round(a / step) * step * _pow2_64(e)).flatten(1)[:, :width]


def exact(case, seed):
    if case["op"] == "sample":
        return None  # whole numbers
    st = prepare(case, seed)
    if case["op"] == "linear":
        x, w = _values64(st["x_codes"], st["x_scales"]), _values64(st["w_codes"], st["w_scales"])
        return x @ w.T
    if case["op"] == "lora":
        out = st["y"].double()
        for i in range(case["adapters"]):
            at = (st["ids"] == i).nonzero()[:, 0]
            t = st["x"][at].double() @ st["a"][i].double().T
            out[at] += st["scale"][i].double() * (t @ st["b"][i].double().T)
        return out
    live = _positions(case)
    if case["op"] == "quant":
        if case["gate"]:
            return None  # a product next to a border of the 8-bit rounding has no one value in 64 bits
        out = _round64(st["x"])
        out[live:] = 0
        return [out]
    h = st["h"].double()
    if case["delta"]:
        h = h + st["delta"].double()
    h[live:] = 0
    outs = [h] if case["delta"] else []
    if case["out"] != "mx8":
        x = h.to(st["h"].dtype).double()
        outs.append(x / torch.sqrt((x * x).sum(1, keepdim=True) / x.shape[1] + EPS) * st["w"].double())
    return outs + [None] * (case["out"] != "y") if outs else None
