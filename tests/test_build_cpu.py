"""What the build makes and when it makes it again (no GPU, no compiler: commands are recorded)."""
import importlib.util
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Commands:
    """Stands in for subprocess.run: notes each command and makes its output file; `fails`: a file name in the command
    of the one that does not compile."""

    def __init__(self, fails=None):
        self.ran, self.fails = [], fails

    def __call__(self, cmd, **kw):
        self.ran.append(cmd)
        if self.fails and any(str(c).endswith(self.fails) for c in cmd):
            return subprocess.CompletedProcess(cmd, 1, "", "does not compile")
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("made")
        return subprocess.CompletedProcess(cmd, 0, "", "")


@pytest.fixture()
def build(monkeypatch, tmp_path):
    from paper_2607_03574_gb300 import build as b
    monkeypatch.setattr(b, "OUT_DIR", str(tmp_path))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libndvm.so"))
    monkeypatch.setattr(b, "TORCH_OPS", str(tmp_path / "ndvm_torch.so"))
    monkeypatch.setattr(b, "_nvcc", lambda: "/usr/local/cuda/bin/nvcc")
    return b


def _commands(monkeypatch, **kw):
    c = Commands(**kw)
    monkeypatch.setattr(subprocess, "run", c)
    return c


def _without_torch(monkeypatch):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))


def test_library_is_built_without_torch(build, monkeypatch):
    """The C ABI and the numpy calls need no PyTorch."""
    _without_torch(monkeypatch)
    c = _commands(monkeypatch)
    assert build.build() == build.LIB and os.path.exists(build.LIB) and not os.path.exists(build.TORCH_OPS)
    assert not any("torch_ops" in str(a) for cmd in c.ran for a in cmd)
    made = len(c.ran)
    assert not build._stale() and build.build() == build.LIB and len(c.ran) == made


def test_library_is_there_where_the_torch_module_does_not_compile(build, monkeypatch):
    """(As with a PyTorch that has no CUDA headers.)  An explicit build says so; loading the library does not ask."""
    c = _commands(monkeypatch, fails="torch_ops.cpp")
    with pytest.raises(RuntimeError, match="torch_ops.cpp failed"):
        build.build()
    assert os.path.exists(build.LIB) and not build._stale()
    c.ran.clear()
    assert build.build(torch_ops=False) == build.LIB and not c.ran


def test_both_are_built_where_torch_is(build, monkeypatch):
    c = _commands(monkeypatch)
    build.build()
    assert os.path.exists(build.LIB) and os.path.exists(build.TORCH_OPS)
    c.ran.clear()
    build.build()
    assert not c.ran
    os.remove(build.TORCH_OPS)
    build.build()
    assert len(c.ran) == 2 and not any(str(a).endswith(".cu") for cmd in c.ran for a in cmd)  # the module alone


def test_programs_are_traced_without_torch(ndvm):
    """Loading the library neither imports PyTorch nor wants the module built against it."""
    code = ("import importlib.util, sys\n"
            "find = importlib.util.find_spec\n"
            "importlib.util.find_spec = lambda name, *a: None if name == 'torch' else find(name, *a)\n"
            "sys.modules['torch'] = None\n"
            "from paper_2607_03574_gb300 import build\n"
            "build.TORCH_OPS = '/nowhere/ndvm_torch.so'\n"
            "build.build = lambda *a, **k: sys.exit('built again')\n"
            "import paper_2607_03574_gb300 as nd\n"
            "print(nd.trace_build('(model (params a b) (* a b))').info()['n_params'])\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "2", (r.stdout, r.stderr)


def test_module_is_made_again_for_another_torch(build, monkeypatch, tmp_path):
    """A module built against one PyTorch may not be loaded into another, however old its sources are."""
    c = _commands(monkeypatch)
    for version in ("2.0", "2.1"):
        root = tmp_path / "torch"
        root.mkdir(exist_ok=True)
        (root / "version.py").write_text(f"__version__ = '{version}'\n")
        monkeypatch.setattr(build, "_torch_root", lambda: str(root))
        assert build._torch_ops_stale()
        c.ran.clear()
        build.build()
        assert any(str(a).endswith("torch_ops.cpp") for cmd in c.ran for a in cmd) and not build._torch_ops_stale()
    monkeypatch.setattr(build, "_torch_root", lambda: str(tmp_path / "elsewhere"))
    assert build._torch_ops_stale()
