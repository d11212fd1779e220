"""The marshalling module depends on the C++ interfaces of one interpreter and one torch; nothing else of the package
does.  Without a usable one the package imports, all other calls work and the ten that need it say what is
missing; the build compiles it again when torch has changed, and leaves it out where there is no torch."""
import importlib.util
import os
import subprocess
import sys

import pytest

import paper_2310_10537_b200 as mx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2310_10537_b200")
USE = """
import sys
sys.path.insert(0, sys.argv[1])
import paper_2310_10537_b200 as mx
assert mx.LIB_PATH.startswith(sys.argv[1])
assert mx.mx_elems_bytes([4, 64], 1, mx.MX_E4M3) == 256 and mx.mx_moe_rows(16, 8, 64, 64) == 4160
print("imported")
try:
    mx.mx_route(None, 2)
except ImportError as e:
    print(e)
"""


def _package_copy(tmp_path):
    pkg = tmp_path / "paper_2310_10537_b200"
    pkg.mkdir()
    for f in ("__init__.py", "binding.py", "build.py"):
        (pkg / f).write_text(open(os.path.join(PKG, f)).read())
    os.symlink(mx.LIB_PATH, pkg / "libmx_b200.so")
    return pkg


@pytest.mark.parametrize("module", [None, b"not a library"])
def test_the_rest_of_the_package_works_without_it(tmp_path, module):
    pkg = _package_copy(tmp_path)
    if module is not None:
        (pkg / "_py_call.so").write_bytes(module)
    p = subprocess.run([sys.executable, "-c", USE, str(tmp_path)], capture_output=True, text=True)
    assert p.returncode == 0, p.stderr
    assert p.stdout.startswith("imported") and "build.py" in p.stdout and "_py_call.so" in p.stdout


def test_a_module_for_another_torch_is_not_used(tmp_path):
    pkg = _package_copy(tmp_path)
    os.symlink(os.path.join(PKG, "_py_call.so"), pkg / "_py_call.so")
    p = subprocess.run([sys.executable, "-c", "import torch\ntorch.__version__ = '0.0.1'\n" + USE, str(tmp_path)], capture_output=True, text=True)
    assert p.returncode == 0, p.stderr
    assert p.stdout.startswith("imported") and "compiled for python" in p.stdout and "0.0.1" in p.stdout


def _build_module():
    spec = importlib.util.spec_from_file_location("_mx_build_under_test", os.path.join(PKG, "build.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_the_build_follows_torch(monkeypatch):
    mod, built = _build_module(), []
    monkeypatch.setattr(mod, "_build_py_call", lambda: built.append(1))
    monkeypatch.setattr(mod, "_compile", lambda *a: pytest.fail("a kernel file was compiled"))
    monkeypatch.setattr(mod.shutil, "which", lambda name: "/usr/bin/" + name)
    assert mod.build() == mod.LIB and not built
    monkeypatch.setattr(mod, "py_call_for", lambda: "python 3.99, torch 0.0.1")
    assert mod.build() == mod.LIB and built == [1]
    monkeypatch.setattr(mod, "py_call_for", lambda: "")  # no torch: the C library is all there is to build
    monkeypatch.setattr(mod, "PY_CALL", mod.PY_CALL + ".absent")
    assert mod.build() == mod.LIB and built == [1]


def test_a_shipped_library_without_a_compiler_is_taken(monkeypatch):
    mod = _build_module()
    monkeypatch.setattr(mod, "PY_CALL", mod.PY_CALL + ".absent")
    monkeypatch.setattr(mod, "_newest_source", lambda: float("inf"))
    monkeypatch.setattr(mod.shutil, "which", lambda name: None)
    assert mod.build() == mod.LIB
