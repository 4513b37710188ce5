"""What a build makes, and what it needs for that: the library needs the HIP compiler alone."""
import os

import pytest

from paper_2606_27866_amd import build


@pytest.fixture
def made(monkeypatch, tmp_path):
    """A build whose compilers write an empty file; the outputs in order."""
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "TENSORS", str(tmp_path / "_tensors.so"))
    out = []

    class Done:
        returncode, stdout, stderr = 0, "", ""

    def run(cmd, **_):
        to = cmd[cmd.index("-o") + 1]
        open(to, "w").close()
        out.append(os.path.basename(to).split(".")[0])
        return Done

    monkeypatch.setattr(build.subprocess, "run", run)
    return out


def test_library_first_then_the_module(made):
    assert build.build() == build.LIB
    assert made == ["lib", "_tensors"]
    assert not build.is_stale()


@pytest.mark.parametrize("lost", ["g++", "torch", "headers"])
def test_library_without_what_only_the_module_needs(made, monkeypatch, capsys, tmp_path, lost):
    if lost == "g++":
        monkeypatch.setattr(build.shutil, "which", lambda name: None)
    elif lost == "torch":
        monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: None)
    else:
        class Spec:
            origin = str(tmp_path / "torch" / "__init__.py")
        monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: Spec)
    assert build.build() == build.LIB and os.path.exists(build.LIB)
    assert made == ["lib"] and lost in capsys.readouterr().err
    assert not build.is_stale()  # nothing that a build here could add


def test_a_failed_module_leaves_the_library(made, monkeypatch):
    """Where the module can be built, its failure is the build's; the library is in its place by then."""
    def fails():
        raise RuntimeError("g++ failed")

    monkeypatch.setattr(build, "build_tensors", fails)
    with pytest.raises(RuntimeError):
        build.build()
    assert made == ["lib"] and os.path.exists(build.LIB) and build.is_stale()
