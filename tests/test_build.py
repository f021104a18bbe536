"""The in-tree build: what it needs, and when it has to run again."""
import os
import subprocess
import sys

import pytest

from paper_2301_01333_b200 import build as B


@pytest.fixture
def elsewhere(monkeypatch, tmp_path):
    """The CUDA library up to date, the torch side missing (in a place of its own: the real one stays as it is)."""
    B.build()
    monkeypatch.setattr(B, "TORCH_LIB", str(tmp_path / "_serving.so"))
    monkeypatch.setattr(B, "_stale", lambda: False)
    return tmp_path


def test_without_a_compiler_for_the_torch_side_the_library_is_built_all_the_same(elsewhere, monkeypatch, capsys):
    monkeypatch.setenv("PATH", str(elsewhere))
    assert B.build() == B.LIB
    assert "g++" in capsys.readouterr().err and not os.path.exists(B.TORCH_LIB)


def test_without_torch_the_library_is_built_all_the_same(elsewhere, monkeypatch, capsys):
    for name in [m for m in sys.modules if m == "torch.utils.cpp_extension"]:
        monkeypatch.delitem(sys.modules, name)
    monkeypatch.setitem(sys.modules, "torch", None)              # importing it raises ImportError
    assert B.build() == B.LIB
    assert "torch" in capsys.readouterr().err and not os.path.exists(B.TORCH_LIB)


def test_the_library_loads_without_the_torch_side(tmp_path):
    """The C interface's binding in a process that cannot import torch."""
    B.build()
    code = "import sys; sys.modules['torch'] = None\nfrom paper_2301_01333_b200 import binding\nprint(binding.gc_version())"
    r = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(B.HERE), capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip(), r.stderr


def test_a_mistake_in_the_torch_side_still_fails_the_build(elsewhere, monkeypatch):
    bad = elsewhere / "bad.cpp"
    bad.write_text("this is not C++\n")
    monkeypatch.setattr(B, "TORCH_SOURCE", str(bad))
    with pytest.raises(RuntimeError):
        B.build()


def test_the_torch_side_is_compiled_again_for_another_torch(monkeypatch):
    import importlib.metadata
    B.build()
    assert not B._torch_stale()
    real = importlib.metadata.version
    monkeypatch.setattr(importlib.metadata, "version", lambda name: "9.9.9" if name == "torch" else real(name))
    assert B._torch_stale()


def test_the_torch_side_says_what_it_was_compiled_for():
    import importlib.metadata
    B.build()
    from paper_2301_01333_b200 import _serving
    assert importlib.metadata.version("torch") in _serving.abi
