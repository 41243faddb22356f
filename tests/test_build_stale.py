"""When the native marshalling module is rebuilt: it is bound to the torch (and Python) it was compiled against."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2306_06098_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def module(tmp_path, monkeypatch):
    """A freshly built module, as far as the files tell; returns a list that counts compilations."""
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / "_marshal.so"))
    calls = []

    def compile_it(cmd, check):
        calls.append(cmd)
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("module")

    monkeypatch.setattr(build.subprocess, "run", compile_it)
    build.build_marshal()
    assert len(calls) == 1 and os.path.exists(build.MARSHAL)
    return calls


def test_it_is_kept_while_nothing_changes(module):
    build.build_marshal()
    assert len(module) == 1
    build.build_marshal(force=True)
    assert len(module) == 2


def test_another_torch_means_another_build(module, monkeypatch):
    monkeypatch.setattr(build, "_bound_to", lambda: "torch 9.9.9, Python 3.12")
    build.build_marshal()
    assert len(module) == 2
    build.build_marshal()
    assert len(module) == 2


def test_a_module_of_unknown_origin_is_rebuilt(module):
    for name in os.listdir(os.path.dirname(build.MARSHAL)):
        if name != "_marshal.so":
            os.remove(os.path.join(os.path.dirname(build.MARSHAL), name))
    build.build_marshal()
    assert len(module) == 2


def test_it_knows_the_torch_that_runs():
    import torch
    assert torch.__version__ in build._bound_to()


def test_a_module_that_does_not_load_says_what_to_do(tmp_path):
    src = os.path.join(ROOT, "paper_2306_06098_b200")
    pkg = tmp_path / "paper_2306_06098_b200"
    (pkg / "csrc").mkdir(parents=True)
    for name in os.listdir(src):
        if name.endswith(".py"):
            shutil.copy(os.path.join(src, name), pkg)
    os.symlink(os.path.join(src, "csrc", "libefcp.so"), pkg / "csrc" / "libefcp.so")
    (pkg / "_marshal.so").write_text("built for another interpreter")
    out = subprocess.run([sys.executable, "-c", "import paper_2306_06098_b200.binding"], cwd=tmp_path, capture_output=True, text=True,
                         timeout=300, env=dict(os.environ, PYTHONPATH=str(tmp_path)))
    assert out.returncode != 0 and "ImportError" in out.stderr
    assert "python -m paper_2306_06098_b200.build" in out.stderr
