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
        blib._here(torch.zeros(3, dtype=torch.int32), "pos", torch.int32, 0)
    with pytest.raises(TypeError, match="device"):
        blib._heads(torch.zeros(3, 2, 64), "q", torch.float32, 0, (3, 2, 64))
