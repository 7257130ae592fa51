"""The token operators' compiled module: what the package needs to be imported, which module is loaded and when it is built (CPU)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def python(code, **kw):
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=600, **kw)


def test_the_package_and_the_c_library_need_no_torch():
    r = python("import sys; sys.modules['torch'] = None\n"
               "import paper_1707_00424_b200 as pb\n"
               "assert pb.lib().parle_strerror(-1) and pb.embedding_grad_workspace_bytes(1, 2000, 10, 4) > 0\n"
               "print(pb.TOP_MAX)")
    assert r.returncode == 0 and r.stdout.strip() == "32", r.stderr
