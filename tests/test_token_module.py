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


def test_built_files_are_loaded_without_their_sources(tmp_path):
    import shutil
    here = copy_of_the_package(tmp_path)
    shutil.rmtree(here / "include")
    shutil.rmtree(here / "paper_1707_00424_b200" / "csrc")
    assert load_in(here) == "loaded"
    r = subprocess.run([sys.executable, "-c", LOAD % "torch.__version__ = '0.1'"], cwd=here, capture_output=True, text=True, timeout=600)
    assert r.returncode != 0 and "torch 0.1" in r.stderr


BUILD = """
import os, sys, time
sys.path.insert(0, '.')
from paper_1707_00424_b200 import build
def slowly(cmd):                                          # a compiler that writes its output in two halves
    with open('compiled', 'a') as f:
        f.write(os.path.basename(cmd[0]) + chr(10))
    stamp = [c for c in cmd if 'BUILT_FROM' in c]
    with open(cmd[cmd.index('-o') + 1], 'wb') as f:
        f.write(b'first half ')
        f.flush()
        time.sleep(1.0)
        f.write((build.module_stamp() if stamp else 'library').encode() + b' second half')
    return ''
build._run = slowly
build.%s()
"""


def build_at_once(here, what, target, ranks=3):
    """Several processes build; what a reader saw of the file meanwhile, and how often it was compiled."""
    import time
    path, seen = here / "paper_1707_00424_b200" / target, set()
    path.unlink()
    running = [subprocess.Popen([sys.executable, "-c", BUILD % what], cwd=here, stderr=subprocess.PIPE, text=True) for _ in range(ranks)]
    while any(p.poll() is None for p in running):
        if path.exists():
            seen.add(path.read_bytes()[-11:])
        time.sleep(0.01)
    assert [p.returncode for p in running] == [0] * ranks, [p.stderr.read() for p in running]
    compiled = (here / "compiled").read_text().split()
    (here / "compiled").unlink()
    left = [f for f in os.listdir(here / "paper_1707_00424_b200") if ".so" in f and f not in ("_token_ops.so", "libparle.so")]
    return seen, compiled, left


def test_processes_that_build_at_once_build_once_and_never_show_half_a_file(tmp_path):
    here = copy_of_the_package(tmp_path)
    for what, target in (("build_module", "_token_ops.so"), ("build", "libparle.so")):
        seen, compiled, left = build_at_once(here, what, target)
        assert seen <= {b"second half"} and len(compiled) == 1 and not left, (seen, compiled, left)


def test_a_failed_build_leaves_the_old_file(tmp_path):
    here = copy_of_the_package(tmp_path)
    for what, target in (("build_module", "_token_ops.so"), ("build", "libparle.so")):
        path = here / "paper_1707_00424_b200" / target
        before = path.read_bytes()
        code = BUILD.replace("time.sleep(1.0)", "raise RuntimeError('no')") % (what + "(force=True) or print")
        r = subprocess.run([sys.executable, "-c", code], cwd=here, capture_output=True, text=True, timeout=600)
        assert r.returncode != 0 and "RuntimeError: no" in r.stderr and path.read_bytes() == before
        assert sorted(f for f in os.listdir(here / "paper_1707_00424_b200") if f.endswith(".so")) == ["_token_ops.so", "libparle.so"]


def test_workspace_of_sizes_beyond_the_c_types_is_that_of_invalid_ones():
    import paper_1707_00424_b200 as pb
    size = pb.embedding_grad_workspace_bytes
    assert size(1, 2000, 10, 4) > 0
    for wrong in ((1 + (1 << 32), 2000, 10, 4), (1, 2000 + (1 << 64), 10, 4), (1, 2000, 10 + (1 << 32), 4), (1, 2000, 10, 4 + (1 << 32)), (1, -1, 10, 4), (1 - (1 << 32), 2000, 10, 4)):
        assert size(*wrong) == 0, wrong
