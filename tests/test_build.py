"""The library's build where what only the torch binding needs is missing."""
import os
import subprocess
import sys

import pytest

from paper_2609_33614_gb300 import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture
def apart(tmp_path, monkeypatch):
    """A build directory of the test's own, with the repository's library in it."""
    build.build()
    for name in ("LIB", "BINDING"):
        monkeypatch.setattr(build, name, str(tmp_path / os.path.basename(getattr(build, name))))
    monkeypatch.setattr(build, "BUILD", str(tmp_path))
    (tmp_path / "libeat.so").write_bytes(b"library")
    (tmp_path / "libeat.stamp").write_text(build._stamp())
    return tmp_path


@pytest.mark.parametrize("missing", ["torch", "headers", "python", "compiler"])
def test_library_without_the_binding(apart, monkeypatch, missing):
    (apart / "_eatops.so").write_bytes(b"of an older library")
    if missing == "torch":
        monkeypatch.setitem(sys.modules, "torch", None)
        word = "torch"
    elif missing == "headers":
        torch = pytest.importorskip("torch")
        monkeypatch.setattr(torch, "__file__", str(apart / "torch" / "__init__.py"))
        word = "Tensor.h"
    elif missing == "python":
        monkeypatch.setattr(build.sysconfig, "get_paths", lambda: {"include": str(apart)})
        word = "Python.h"
    else:
        monkeypatch.setenv("CXX", str(apart / "no-such-compiler"))
        word = "compiler"
    with pytest.warns(UserWarning, match="_eatops.so is not built") as seen:
        assert build.build() == str(apart / "libeat.so")
    assert any(word in str(w.message) for w in seen)
    assert not (apart / "_eatops.so").exists()


def test_a_binding_that_does_not_compile_is_an_error(apart, monkeypatch):
    monkeypatch.setenv("CXX", "false")
    with pytest.raises(RuntimeError, match="failed on"):
        build.build(force=False)


def test_functions_of_tensors_say_what_is_missing(tmp_path):
    code = ("from paper_2609_33614_gb300 import eat; eat.PKG = %r\n"
            "try:\n    eat.rms_norm(None, None)\n"
            "except RuntimeError as e:\n    assert '_eatops.so' in str(e)\n"
            "else:\n    raise SystemExit(1)\n") % str(tmp_path)
    r = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(HERE),
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
