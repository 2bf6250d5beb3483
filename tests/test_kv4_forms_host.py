"""Which form and how many chunks a call of paged 4-bit attention takes, asked of
the library without a device: the shapes of the device tests reach the kernels
that they are meant for."""
import ctypes as C

import pytest
import torch

from paper_2606_09514_amd import lib as blib
from test_kv4_attention_gpu import PROMPTS, chunks_are


class Shape:
    """What a cache and a call's sizes say; no memory behind it."""

    def __init__(self, nq, nkv, hd, page, pages=100):
        self.struct = blib.KV4Struct(16, 16, 16, 16, pages, page, nkv, hd)
        self.nq, self.hd = nq, hd

    def form(self, dtype, n_rows, B, max_rows, max_len):
        return blib.kv4_attention_form(self, dtype, self.nq, n_rows, B, max_rows, max_len)

    def workspace(self, n_rows, B, max_rows, max_len):
        return blib.kv4_attention_workspace(self, self.nq, n_rows, B, max_rows, max_len)


def test_prompt_shapes_take_the_prompt_form():
    for lens, news, nq, nkv, hd, page, chunks in PROMPTS:
        s = Shape(nq, nkv, hd, page)
        parts, n = s.form(torch.bfloat16, sum(news) + 3, len(lens), max(news), max(lens))
        assert parts == 1 and chunks_are(n, chunks), (lens, news, n)
    # every page size and head size, one KV head and more, few and many (row, head) pairs to join
    assert {c[5] for c in PROMPTS} == {16, 32, 64, 128, 256}
    assert {(c[4], c[6]) for c in PROMPTS} == {(h, n) for h in (64, 128) for n in ("one", "few", "many")}
    assert {(sum(c[1]) + 3) * c[2] > 4096 for c in PROMPTS if c[6] == "few"} == {True, False}


def test_weights_of_single_tokens_and_of_fp32_calls():
    s = Shape(32, 8, 128, 64)
    for B, n, length in ((1, 1, 2048), (96, 1, 2048), (3, 16, 100), (1, 1, 0)):
        assert s.form(torch.bfloat16, B * n, B, n, length)[0] == 2          # 64 columns and fewer
    for n in (1, 1024):
        assert s.form(torch.float32, n, 1, n, 8000)[0] == 3
    assert s.form(torch.bfloat16, 0, 0, 1, 100) == (2, 1)


def test_form_refuses_what_the_call_refuses():
    a = blib.KV4Attn(n_heads=32, n_rows=1, max_rows=1, max_len=100, dtype=blib.BF16)
    cache = blib.KV4Struct(16, 16, 16, 16, 4, 64, 8, 128)
    ask = lambda c, x, B: blib.lib().buddy_kv4_attention_form(C.byref(c), C.byref(x) if x else None, B, None, None)
    assert ask(cache, a, 1) == blib.OK and ask(cache, None, 1) == blib.EINVAL and ask(cache, a, -1) == blib.EINVAL
    assert ask(cache, a, 1025) == blib.ECAPACITY
    a.n_heads = 30
    assert ask(cache, a, 1) == blib.ESHAPE
    with pytest.raises(TypeError):
        Shape(32, 8, 128, 64).form(torch.float16, 1, 1, 1, 100)
    with pytest.raises(blib.BuddyError):
        Shape(32, 8, 96, 64).form(torch.bfloat16, 1, 1, 1, 100)


def test_a_workspace_is_enough_for_every_smaller_step():
    """What a call of fewer rows, sequences or shorter ones asks for, and what
    it writes, fits the workspace of the larger one; of either type."""
    import random
    rng = random.Random(3)
    log = lambda hi: int(2 ** rng.uniform(0, hi))
    split = 0
    for _ in range(4000):
        nkv, G, hd = rng.choice([1, 2, 3, 8, 40]), rng.choice([1, 4, 7, 16]), rng.choice([64, 128])
        s = Shape(nkv * G, nkv, hd, 64)
        rows, B, length = log(13), log(9), log(17)
        big = s.workspace(rows, B, rng.randint(1, rows), length)
        assert 16 <= big <= 2 ** 17 * (hd + 2) * 4
        rows, B, length = rng.randint(1, rows), rng.randint(1, B), rng.randint(0, length)
        max_rows = rng.randint(1, rows)
        assert s.workspace(rows, B, max_rows, length) <= big
        for dtype in (torch.bfloat16, torch.float32):
            chunks = s.form(dtype, rows, B, max_rows, length)[1]
            assert chunks == 1 or rows * nkv * G * chunks * (hd + 2) * 4 <= big
            split += chunks > 1
    assert split > 2000
    # a batch of single tokens that ends, request after request
    s = Shape(32, 8, 128, 64)
    for length in (2048, 4096, 120000):
        big = s.workspace(96, 96, 1, length)
        for B in range(1, 97):
            assert s.workspace(B, B, 1, length) <= big and s.workspace(96, B, 1, length) <= big
    # many rows and heads: not split at all
    assert s.form(torch.float32, 5000, 1, 1, 120000)[1] == 1 and s.form(torch.float32, 5, 1, 1, 120000)[1] > 60
