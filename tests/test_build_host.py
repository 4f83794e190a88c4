"""The build of the library and of the module beside it: the library does not
depend on what only the module needs."""
import os
import subprocess
import sys

import pytest

from paper_2504_11320_amd import build as Bd


@pytest.fixture
def fake(monkeypatch, tmp_path):
    """Builds into a folder of its own; compilers write empty files, or fail
    where `fails` says so."""
    lib, module = str(tmp_path / "lib.so"), str(tmp_path / "module.so")
    ran, fails = [], []

    def run(cmd, check=True, **kw):
        out = cmd[cmd.index("-o") + 1]
        ran.append(out)
        if any(out.startswith(f) for f in fails):
            raise subprocess.CalledProcessError(1, cmd)
        open(out, "w").close()

    monkeypatch.setattr(Bd, "LIB", lib)
    monkeypatch.setattr(Bd, "BINDING", module)
    monkeypatch.setattr(Bd.subprocess, "run", run)
    return lib, module, ran, fails


def test_both_are_built(fake):
    lib, module, ran, _ = fake
    assert Bd.build(out=lib) == lib
    assert os.path.exists(lib) and os.path.exists(module)
    assert len(ran) == len(Bd.SRCS) + 2


def test_module_that_does_not_compile(fake):
    """An error, but the library is there, and no module of an earlier build."""
    lib, module, _, fails = fake
    open(module, "w").close()
    fails.append(module)
    with pytest.raises(subprocess.CalledProcessError):
        Bd.build(out=lib)
    assert os.path.exists(lib) and not os.path.exists(module)


@pytest.mark.parametrize("lacks", ["torch", "compiler", "headers"])
def test_without_what_the_module_needs(fake, monkeypatch, capsys, lacks):
    """The library alone, as without the module's sources; what is lacking is
    said."""
    lib, module, ran, _ = fake
    open(module, "w").close()
    if lacks == "torch":
        monkeypatch.setitem(sys.modules, "torch", None)
    elif lacks == "compiler":
        monkeypatch.setenv("CXX", "/nowhere/c++")
    else:
        monkeypatch.setattr(Bd.sysconfig, "get_path", lambda name: "/nowhere")
    assert Bd.build(out=lib) == lib
    assert os.path.exists(lib) and not os.path.exists(module)
    assert len(ran) == len(Bd.SRCS) + 1
    assert "kv.py" in capsys.readouterr().err


def test_other_libraries_come_alone(fake, tmp_path):
    _, module, ran, _ = fake
    other = str(tmp_path / "other.so")
    Bd.build(out=other)
    assert os.path.exists(other) and not os.path.exists(module)
    assert len(ran) == len(Bd.SRCS) + 1
