"""What is built when, and what is refused at loading (no GPU needed)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_library_needs_no_torch(tmp_path):
    """The C interface is built without torch; its binding is left out."""
    from paper_2607_27692_b200 import build
    build.build()
    code = f"""
import sys
sys.modules["torch"] = None                     # as if it were not installed
from paper_2607_27692_b200 import build
build.BINDING_PATH = {str(tmp_path / "_paged.so")!r}
build.BINDING_STAMP = build.BINDING_PATH + ".stamp"
print(build.build())
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert r.stdout.strip() == build.LIB_PATH and not os.listdir(tmp_path)
