"""The operators around attention without a device: refusals of their entry
points, scales and workspaces, in a build of the host code under
AddressSanitizer and UndefinedBehaviorSanitizer; the binding's own checks; the
fragment reads that the projection issues through inline asm."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

from test_asm_guards import device_asm, hazards
from test_sanitizers import CSRC, ENV, HIPCC, HOST_SAN, SAN, run

FLAGS = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xarch_device", "-O1", "-Xarch_device", "-g0",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", *HOST_SAN]


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_host_code_under_address_and_ub_sanitizers(tmp_path):
    objs, procs = [], []
    for src in (os.path.join(CSRC, "rows8.hip"), os.path.join(CSRC, "lora.hip"), os.path.join(CSRC, "sample.hip"),
                os.path.join(SAN, "serving_driver.cpp")):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        objs.append(obj)
        procs.append(subprocess.Popen([HIPCC, *FLAGS, "-x", "hip", "-c", src, "-o", obj],
                                      stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
    for p in procs:
        out, _ = p.communicate()
        assert p.returncode == 0, out[-4000:]
    exe = str(tmp_path / "serving_driver")
    run([HIPCC, "--offload-arch=gfx950", *HOST_SAN[:4], *objs, "-o", exe])
    env = dict(ENV, ASAN_OPTIONS=ENV["ASAN_OPTIONS"] + ":detect_leaks=0")
    r = run([exe], env=env)
    assert r.stdout.strip().endswith("serving driver ok"), r.stdout


def test_binding_refuses_host_tensors_and_other_shapes():
    from paper_2606_09514_amd import lib as blib
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    with pytest.raises(TypeError, match="codes: expected a uint8 device tensor"):
        blib.MX8(u8(3, 48), u8(3, 16))
    f = lambda *s: torch.zeros(s)
    for a, b in ((f(2, 8, 16), f(3, 16, 8)), (f(2, 8, 16), f(2, 16, 16)), (f(8, 16), f(2, 16, 8))):
        with pytest.raises(ValueError, match="expected a"):
            blib.Adapters(a, b, f(2))
    with pytest.raises(ValueError, match="scale: expected 2"):
        blib.Adapters(f(2, 8, 16), f(2, 16, 8), f(1))
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        blib.Adapters(f(2, 8, 16).half(), f(2, 16, 8).half(), f(2))
    with pytest.raises(TypeError, match="device"):
        blib.Adapters(f(2, 8, 16), f(2, 16, 8), f(2))


def test_sizes_that_are_refused_have_no_workspace():
    from paper_2606_09514_amd import lib as blib
    with pytest.raises(ValueError, match="refuses"):
        blib.sample_workspace(3, 0)
    with pytest.raises(ValueError, match="refuses"):
        blib.lora_plan_size(3, 5000)
    assert blib.sample_workspace(0, 7) >= 16 and blib.lora_plan_size(1, 1) >= 4


def test_compiled_marshalling_refuses_what_is_not_a_tensor_of_the_device():
    """Called as the binding calls it, without a device: the checks come before
    anything is passed on."""
    from paper_2606_09514_amd import lib as blib
    b = blib.bind()
    f, i32 = (lambda *s: torch.zeros(s)), (lambda *s: torch.zeros(s, dtype=torch.int32))
    u8 = torch.zeros(64, dtype=torch.uint8)
    m = blib.MX8Struct(None, None, 48, 16, 3, 48)
    l = blib.LoraStruct(None, None, None, blib.F32, 2, 8, 16, 24)
    here = "expected a tensor on the current device"
    with pytest.raises(TypeError, match="h: " + here):
        b.add_rmsnorm(f(3, 48), f(48), None, None, f(3, 48), None, None, 1e-6, 0, 0)
    with pytest.raises(TypeError, match="weight: expected a tensor"):
        b.add_rmsnorm(f(3, 48), None, None, None, f(3, 48), None, None, 1e-6, 0, 0)
    with pytest.raises(ValueError, match="rows"):
        b.add_rmsnorm(f(48), f(48), None, None, f(48), None, None, 1e-6, 0, 0)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        b.add_rmsnorm(f(3, 48).half(), f(48), None, None, f(3, 48), None, None, 1e-6, 0, 0)
    with pytest.raises(TypeError, match="x: " + here):
        b.mx8_quantize(f(3, 48), C.addressof(m), None, None, 0, 0)
    with pytest.raises(TypeError, match="out: " + here):
        b.mx8_read(C.addressof(m), f(3, 48), 0, 0)
    with pytest.raises(TypeError, match="out: " + here):
        b.mx8_linear(C.addressof(m), C.addressof(m), f(3, 3), u8, 0, 0)
    with pytest.raises(TypeError, match="ids: " + here):
        b.lora_plan(i32(3), 2, i32(200), 0, 0)
    with pytest.raises(TypeError, match="x: " + here):
        b.lora_add(C.addressof(l), f(3, 16), f(3, 24), f(3, 24), i32(200), u8, 0, 0)
    with pytest.raises(TypeError, match="logits: " + here):
        b.sample(f(3, 48), f(3), i32(3), u8, f(3), None, None, None, 0, 0)
    for name in ("add_rmsnorm", "mx8_quantize", "mx8_read", "mx8_linear", "lora_plan", "lora_add", "sample"):
        with pytest.raises(TypeError, match="number of arguments"):
            getattr(b, name)(1, 2)


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_no_register_of_an_asm_read_is_touched_before_its_wait():
    """The projection of many rows reads its fragments from LDS in inline asm
    and waits with an lgkmcnt(0) of its own."""
    asm = device_asm("linear8.hip")
    bodies = {}
    for m in re.finditer(r"^(_ZN5buddy\S*kernel\S*):", asm, re.M):
        bodies[m.group(1)] = asm[m.end():asm.index(".Lfunc_end", m.end())].splitlines()
    tile = [b for k, b in bodies.items() if "11tile_kernel" in k]
    assert len(tile) == 1 and sum(ln.strip().startswith("ds_read_b128") for ln in tile[0]) >= 16
    batch = [b for k, b in bodies.items() if "12batch_kernel" in k]
    assert len(batch) >= 20 and all(sum(ln.strip().startswith("ds_read_b32") for ln in b) >= 4 for b in batch)
    # the walk knows reads of four registers: those of one as such
    wide = lambda b: [re.sub(r"ds_read_b32 v(\d+),", r"ds_read_b128 v[\1:\1],", ln) for ln in b]
    bad = {k: h[:3] for k, b in bodies.items() if (h := hazards(wide(b)))}
    assert not bad, bad
