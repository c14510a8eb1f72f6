"""What build_library() makes where something that it needs is missing.  Nothing is compiled: the compilers' commands are recorded."""
import subprocess
import sys

import pytest

from paper_2603_27156_amd import build


@pytest.fixture
def commands(tmp_path, monkeypatch):
    """A tree of its own and the commands that ran in it; each leaves its output, or fails if its program is in `commands.broken`."""
    for name in ("HERE", "LIB", "MARSHAL"):
        monkeypatch.setattr(build, name, str(tmp_path / {"HERE": "", "LIB": "libgsr.so", "MARSHAL": "libgsr_marshal.so"}[name]))

    class Commands(list):
        broken = None

    ran = Commands()

    def check_call(cmd, **_):
        ran.append(cmd)
        if ran.broken and cmd[0] == ran.broken[0]:
            raise ran.broken[1]
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("built")
        return 0

    monkeypatch.setattr(subprocess, "check_call", check_call)
    monkeypatch.setenv("HIPCC", "hipcc")
    monkeypatch.setenv("CXX", "host-compiler")
    return ran


def test_all_is_there(commands, tmp_path):
    pytest.importorskip("torch")
    assert build.build_library(verbose=False) == str(tmp_path / "libgsr.so")
    assert (tmp_path / "libgsr.so").exists() and (tmp_path / "libgsr_marshal.so").exists()
    assert sum(c[0] == "hipcc" for c in commands) == len(build.SOURCES) + 1 and sum(c[0] == "host-compiler" for c in commands) == 1


@pytest.mark.parametrize("missing", ["torch", "compiler", "headers"])
def test_the_library_is_built_without_the_binding_s_helper(commands, tmp_path, monkeypatch, capsys, missing):
    if missing == "torch":
        monkeypatch.setitem(sys.modules, "torch", None)
    else:
        pytest.importorskip("torch")
        commands.broken = ("host-compiler", FileNotFoundError("host-compiler") if missing == "compiler" else subprocess.CalledProcessError(1, "host-compiler"))
    (tmp_path / "libgsr_marshal.so").write_text("of an earlier build")
    assert build.build_library(verbose=False) == str(tmp_path / "libgsr.so")
    assert (tmp_path / "libgsr.so").exists()
    assert not (tmp_path / "libgsr_marshal.so").exists() and "libgsr_marshal.so" in capsys.readouterr().err


def test_a_kernel_that_does_not_compile_fails_the_build(commands, tmp_path):
    commands.broken = ("hipcc", subprocess.CalledProcessError(1, "hipcc"))
    with pytest.raises(subprocess.CalledProcessError):
        build.build_library(verbose=False)
    assert not (tmp_path / "libgsr.so").exists()
