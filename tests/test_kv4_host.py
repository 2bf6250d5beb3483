"""The paged 4-bit cache without a device: refusals of its entry points and
the kernels' address arithmetic (damaged page ids and slots among them), in a
build of the host code under AddressSanitizer and UndefinedBehaviorSanitizer;
the binding's own checks."""
import os
import subprocess

import pytest
import torch

from test_sanitizers import CSRC, ENV, HIPCC, HOST_SAN, SAN, run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_host_code_and_offsets_under_address_and_ub_sanitizers(tmp_path):
    objs, procs = [], []
    for src in ("kv4.hip", "kv4_attn.hip"):
        obj = str(tmp_path / (src + ".o"))
        objs.append(obj)
        procs.append(subprocess.Popen(
            [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xarch_device", "-O1",
             "-Xarch_device", "-g0", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", *HOST_SAN,
             "-c", os.path.join(CSRC, src), "-o", obj],
            stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
    for p in procs:
        out, _ = p.communicate()
        assert p.returncode == 0, out[-4000:]
    drv = str(tmp_path / "kv4_driver.o")
    run([HIPCC, "-O1", "-g", "-std=c++17", *HOST_SAN, "-c", os.path.join(SAN, "kv4_driver.cpp"), "-o", drv])
    exe = str(tmp_path / "kv4_driver")
    run([HIPCC, "--offload-arch=gfx950", *HOST_SAN[:4], *objs, drv, "-o", exe])
    env = dict(ENV, ASAN_OPTIONS=ENV["ASAN_OPTIONS"] + ":detect_leaks=0")
    r = run([exe], env=env)
    assert r.stdout.strip().endswith("kv4 driver ok"), r.stdout


def test_binding_refuses_host_tensors_and_other_shapes():
    from paper_2606_09514_amd import lib as blib
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    with pytest.raises(ValueError, match="different shapes"):
        blib.KV4(u8(2, 3, 16, 64), u8(2, 3, 16, 64), u8(2, 3, 2, 16), u8(2, 3, 2, 16))
    with pytest.raises(ValueError, match="expected"):
        blib.KV4(u8(2, 3, 16), u8(2, 3, 16), u8(2, 3, 2), u8(2, 3, 2))
    with pytest.raises(TypeError, match="device"):
        blib.KV4(u8(2, 3, 16, 64), u8(2, 3, 16, 64), u8(2, 3, 4, 16), u8(2, 3, 4, 16))


def test_compiled_marshalling_refuses_what_is_not_a_tensor_of_the_device():
    """Called as the binding calls it, without a device: the checks come
    before anything is passed on."""
    from paper_2606_09514_amd import lib as blib
    b = blib.bind()
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    t = i32(2, 4)
    with pytest.raises(TypeError, match="table: expected a tensor on the current device"):
        b.plan_pages(i32(2), i32(2), t, i32(4), i32(2), 16, i32(2), i32(2), i32(3), i32(8), i32(8),
                     torch.zeros(2, dtype=torch.uint8), 0, 0)
    with pytest.raises(TypeError, match="table: expected a tensor"):
        b.release_pages(i32(2), None, 5, i32(4), i32(2), 16, i32(2), i32(2), 0, 0)
    with pytest.raises(TypeError, match="number of arguments"):
        b.kv4_read(1, 2)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        h = torch.zeros((3, 2, 64), dtype=torch.float16)
        b.qk_norm_rope(h, h, i32(3), h, h, None, None, 1e-6, 1e4, None, False, 0, 0)
    with pytest.raises(ValueError, match="rows"):
        f = torch.zeros((3, 64))
        b.qk_norm_rope(f, f, i32(3), f, f, None, None, 1e-6, 1e4, None, False, 0, 0)


def test_marshalling_fails_loudly_without_its_library(monkeypatch):
    import sys

    from paper_2606_09514_amd import lib as blib
    monkeypatch.setattr(blib, "_bind", None)
    monkeypatch.setitem(sys.modules, "paper_2606_09514_amd._kv4_bind", None)
    monkeypatch.delattr(sys.modules["paper_2606_09514_amd"], "_kv4_bind", raising=False)
    with pytest.raises(RuntimeError, match="not built"):
        blib.bind()
