"""What a build makes anew, and what it needs."""
import os
import subprocess
import sys

import pytest

from paper_2604_07609_b200 import binding as B
from paper_2604_07609_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def test_the_library_is_built_without_torch():
    """nvcc is all that libblink.so needs, and what does not touch the operators' tensors works with it."""
    code = ("import sys; sys.modules['torch'] = None\n"
            "from paper_2604_07609_b200 import build, binding\n"
            "build.MARSHAL = build.MARSHAL + '.missing'\n"
            "assert build.build() == build.LIB and binding.lib().blink_strerror(0)\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert "no torch" in r.stderr and not os.path.exists(build.MARSHAL + ".missing")


def test_a_marshaller_for_another_torch_is_built_again(monkeypatch, tmp_path):
    ran = []

    def run(cmd, **kw):
        ran.append(cmd)
        return subprocess.CompletedProcess(cmd, 0, "", "")
    monkeypatch.setattr(build.subprocess, "run", run)
    build.build_marshal()
    assert ran == []                              # fresh
    monkeypatch.setattr(build, "marshal_for", lambda: "torch 0.0, another")
    build.build_marshal()
    assert len(ran) == 1 and '-DBLINK_BUILT_FOR="torch 0.0, another"' in ran[0]


def test_a_marshaller_for_another_torch_is_not_used(monkeypatch):
    assert B._marshal().built == f"built for {build.marshal_for()}."
    monkeypatch.setattr(B, "_marshal_module", None)
    monkeypatch.setattr(build, "marshal_for", lambda: "torch 0.0, another")
    with pytest.raises(RuntimeError, match="torch 0.0, another"):
        B._marshal()


def test_a_torch_that_is_no_installed_package_has_a_version_too(monkeypatch):
    import torch

    def none(name):
        raise build.importlib.metadata.PackageNotFoundError(name)
    monkeypatch.setattr(build.importlib.metadata, "version", none)
    assert build.marshal_for().startswith(f"torch {torch.__version__}, ")
