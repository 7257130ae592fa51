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


def copy_of_the_package(tmp_path):
    """The package with its sources and built files in another place, the library newer than its sources."""
    import shutil
    from paper_1707_00424_b200 import build
    build.build_module()
    here = tmp_path / "copy"
    shutil.copytree(os.path.join(ROOT, "include"), here / "include")
    shutil.copytree(os.path.join(ROOT, "paper_1707_00424_b200"), here / "paper_1707_00424_b200", ignore=shutil.ignore_patterns("__pycache__"))
    os.utime(here / "paper_1707_00424_b200" / "libparle.so")
    return here


LOAD = """
import sys
sys.path.insert(0, '.')
import torch
from paper_1707_00424_b200 import build, token_ops
def compiles(cmd):
    print('compiles', [c for c in cmd if c.endswith('.cpp')])
    sys.exit(0)
build._run = compiles
%s
token_ops.load()
print('loaded')
"""


def load_in(here, before=""):
    r = subprocess.run([sys.executable, "-c", LOAD % before], cwd=here, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr
    return r.stdout.split()[0]


def test_a_module_of_the_same_sources_is_loaded_whatever_the_files_times(tmp_path):
    here = copy_of_the_package(tmp_path)
    os.utime(here / "paper_1707_00424_b200" / "_token_ops.so", (0, 0))
    assert load_in(here) == "loaded"


def test_a_module_of_other_sources_or_for_another_torch_is_built_again(tmp_path):
    here = copy_of_the_package(tmp_path)
    assert load_in(here, "torch.__version__ = '0.1'") == "compiles"
    for changed in (here / "include" / "parle.h", here / "paper_1707_00424_b200" / "csrc" / "token_bindings.cpp"):
        text = changed.read_text()
        changed.write_text(text + "\n")
        for built in ("_token_ops.so", "libparle.so"):    # newer than the change
            os.utime(here / "paper_1707_00424_b200" / built)
        assert load_in(here) == "compiles"
        changed.write_text(text)
