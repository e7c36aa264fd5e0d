"""The build on a box that cannot compile the binding's look at its tensors: the library is built all the same, and no module of an
earlier build stays."""
import os
import subprocess

import pytest

from paper_2506_03762_amd import build


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """A build in a folder of its own by a compiler that writes what it is asked for; `how` is what g++ does."""
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libaha.so"))
    monkeypatch.setattr(build, "TENSORS", str(tmp_path / "_tensors.so"))
    monkeypatch.setattr(build, "OBJDIR", str(tmp_path / "_build"))
    (tmp_path / "_tensors.so").write_text("earlier")

    def with_gxx(how):
        def run(cmd, **kw):
            if cmd[0] == "g++" and how != "works":
                if how == "missing":
                    raise FileNotFoundError(2, "No such file or directory", "g++")
                return subprocess.CompletedProcess(cmd, 1, "", "tensors.cpp:3: fatal error: no such header")
            with open(cmd[cmd.index("-o") + 1], "w") as f:
                f.write("built")
            return subprocess.CompletedProcess(cmd, 0, "", "")
        monkeypatch.setattr(build, "subprocess", type("run", (), {"run": staticmethod(run)}))
        return build.build()
    return with_gxx


@pytest.mark.parametrize("how, why", [("missing", "g++"), ("fails", "no such header")])
def test_without_the_compiled_checks(elsewhere, how, why, capsys):
    lib = elsewhere(how)
    assert open(lib).read() == "built"
    assert not os.path.exists(build.TENSORS)
    said = capsys.readouterr().err
    assert "_tensors" in said and why in said


def test_with_the_compiled_checks(elsewhere, capsys):
    assert open(elsewhere("works")).read() == "built" and open(build.TENSORS).read() == "built"
    assert capsys.readouterr().err == ""


def test_a_kernel_that_does_not_compile_still_ends_the_build(elsewhere, monkeypatch):
    monkeypatch.setattr(build, "SOURCES", ["a.hip"])
    elsewhere("works")
    monkeypatch.setattr(build.subprocess, "run", staticmethod(lambda cmd, **kw: subprocess.CompletedProcess(cmd, 1, "", "error")))
    with pytest.raises(RuntimeError, match="hipcc failed"):
        build.build()
