"""What the build needs: the library and its nets neither a host compiler nor Python's
headers, which only the operators' binding with tensors does."""

import os
import shutil
import subprocess
import sys
import sysconfig

import pytest

from paper_1902_06714_amd import build, nf

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def stage(tmp_path, monkeypatch):
    """The build with commands that only leave their outputs."""
    ran = []

    def run(cmd, verbose):
        ran.append(cmd)
        if stage_fails and any(c.endswith(stage_fails[0]) for c in cmd):
            raise RuntimeError("build step failed")
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write(" ".join(cmd))
    stage_fails = []
    monkeypatch.setattr(build, "_run", run)
    monkeypatch.setattr(build, "ROOT", str(tmp_path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libnf.so"))
    monkeypatch.setattr(build, "BIND", str(tmp_path / "_nfbind.so"))
    (tmp_path / "_nfbind.so").write_text("an earlier build's")
    return ran, stage_fails


def _no_headers(monkeypatch):
    monkeypatch.setattr(sysconfig, "get_paths", lambda *a: {"include": "/nonexistent"})


def _no_compiler(monkeypatch):
    which = shutil.which
    monkeypatch.delenv("CXX", raising=False)
    monkeypatch.setattr(shutil, "which", lambda c, *a: None if os.path.basename(c) in ("g++", "c++", "clang++") else which(c, *a))


def _no_torch(monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)


@pytest.mark.parametrize("lacks", [_no_headers, _no_compiler, _no_torch])
def test_the_library_is_built_without_what_the_binding_needs(stage, monkeypatch, capsys, lacks):
    lacks(monkeypatch)
    assert build.build() == build.LIB and os.path.exists(build.LIB)
    assert not os.path.exists(build.BIND) and not any("nf_bind.cpp" in c for cmd in stage[0] for c in cmd)
    assert "no operators on tensors" in capsys.readouterr().err


def test_the_library_is_there_when_the_binding_fails(stage):
    stage[1].append("nf_bind.cpp")
    with pytest.raises(RuntimeError):
        build.build()
    assert os.path.exists(build.LIB) and not os.path.exists(build.BIND)


def test_the_binding_is_built_with_torchs_abi(stage, monkeypatch):
    import torch
    for abi in (True, False):
        monkeypatch.setattr(torch, "compiled_with_cxx11_abi", lambda: abi)
        build.build()
        assert any(f"-D_GLIBCXX_USE_CXX11_ABI={int(abi)}" in cmd for cmd in stage[0][-20:])
        assert "libtorch" not in open(build.LIB).read() and "-ltorch_python" in open(build.BIND).read()


def test_nets_need_no_binding(tmp_path):
    """The package without _nfbind.so: it is imported, and its operators say what is missing."""
    here = os.path.dirname(nf.LIB_PATH)
    package = tmp_path / "alone"
    package.mkdir()
    (package / "__init__.py").write_text("")
    os.symlink(os.path.join(here, "nf.py"), package / "nf.py")
    os.symlink(nf.LIB_PATH, package / "libnf.so")
    program = """
import torch
from alone import nf
net = None
try:
    net = nf.nf_net_create((7, 3), "relu")
except nf.NfError as e:                        # no GPU here
    assert e.status == nf.NF_EDEVICE, e
assert nf.nf_logprobs_work(nf.NF_F32, 1, 10) == 0
try:
    nf.nf_logprobs(torch.zeros(2, 3))
except ImportError as e:
    print("refused:", e)
"""
    out = subprocess.run([sys.executable, "-c", program], cwd=tmp_path, capture_output=True, text=True,
                         env={**os.environ, "PYTHONPATH": str(tmp_path), "PYTHONDONTWRITEBYTECODE": "1"})
    assert out.returncode == 0, out.stderr
    assert "refused:" in out.stdout and "_nfbind" in out.stdout
