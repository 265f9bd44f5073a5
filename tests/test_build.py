"""What is built when, and what is refused at loading (no GPU needed)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("torch", ["None", "types.SimpleNamespace(version=types.SimpleNamespace(cuda=None), __file__='', __version__='2')"])
def test_the_library_needs_no_torch(tmp_path, torch):
    """The C interface is built without torch, and beside one without CUDA; its binding is left out."""
    from paper_2607_27692_b200 import build
    build.build()
    code = f"""
import sys, types
sys.modules["torch"] = {torch}                  # None: as if it were not installed
from paper_2607_27692_b200 import build
build.BINDING_PATH = {str(tmp_path / "_paged.so")!r}
build.BINDING_STAMP = build.BINDING_PATH + ".stamp"
print(build.build())
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert r.stdout.strip() == build.LIB_PATH and not os.listdir(tmp_path)


def test_a_binding_of_another_torch_is_stale(monkeypatch, tmp_path):
    from paper_2607_27692_b200 import build
    build.build()
    assert not build.binding_is_stale()
    path, stamp = tmp_path / "_paged.so", tmp_path / "_paged.so.stamp"
    path.write_bytes(b"")
    monkeypatch.setattr(build, "BINDING_PATH", str(path))
    monkeypatch.setattr(build, "BINDING_STAMP", str(stamp))
    assert build.binding_is_stale(), "no record of what it was compiled against"
    stamp.write_text(build.binding_target() + "\n")
    assert not build.binding_is_stale()
    for other in ("cpython-399", "torch 0.4.1"):
        stamp.write_text(build.binding_target().replace(build.binding_target().split(" ")[0], other))
        assert build.binding_is_stale()
    monkeypatch.setattr(build, "has_torch", lambda: False)
    assert not build.binding_is_stale()


def test_a_binding_of_another_torch_is_not_used(monkeypatch):
    from paper_2607_27692_b200 import build, paged
    build.build()
    paged._binding()
    monkeypatch.setattr(paged, "_module", None)
    monkeypatch.setattr(build, "binding_target", lambda: "cpython-399 torch 0.4.1 cxx11 0")
    with pytest.raises(paged._rt.RetopkError, match="build it again"):
        paged.Rope(64)
