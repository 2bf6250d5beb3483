"""The build: the library does not depend on its binding."""
import os

import pytest

from paper_2606_09514_amd import build
from test_sanitizers import HIPCC


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
@pytest.mark.parametrize("fault", ["does not compile", "no compiler", "no torch"])
def test_library_is_built_without_its_binding(fault, monkeypatch, tmp_path):
    so, bind = tmp_path / "libbuddy.so", tmp_path / "_kv4_bind.so"
    bind.write_text("of another build")
    monkeypatch.setattr(build, "HERE", str(tmp_path))
    monkeypatch.setattr(build, "SO", str(so))
    monkeypatch.setattr(build, "BIND_SO", str(bind))
    monkeypatch.setattr(build, "SOURCES", ["prior.hip"])

    def command(obj):
        if fault == "no torch":
            raise ImportError("No module named 'torch'")
        return ["false"] if fault == "does not compile" else [str(tmp_path / "no-such-compiler"), obj]

    monkeypatch.setattr(build, "bind_command", command)
    with pytest.raises(RuntimeError, match="binding"):
        build.build()
    assert so.exists() and not bind.exists()
