"""The C library is built with hipcc alone: without torch or Python's headers the
build ends well, without the extension of the decoding calls, which then say so."""
import os
import sysconfig

import pytest

from paper_2006_12645_amd import build as B


@pytest.fixture
def no_compiler(monkeypatch, tmp_path):
    """build() with compilers that do nothing, in a place of its own."""
    calls = []
    monkeypatch.setattr(B, "BUILD", str(tmp_path / "build"))
    monkeypatch.setattr(B, "LIB", str(tmp_path / "libgba.so"))
    monkeypatch.setattr(B, "BINDING", str(tmp_path / "_gba_decode.so"))
    monkeypatch.setattr(B, "_compile", lambda unit, verbose: str(tmp_path / unit[2]))
    monkeypatch.setattr(B, "_check_no_missing_kernels", lambda lib: None)

    def run(cmd, **kw):
        calls.append(cmd)
        with open(cmd[cmd.index("-o") + 1], "w"):
            pass

    monkeypatch.setattr(B.subprocess, "run", run)
    return calls


def test_with_both(no_compiler):
    pytest.importorskip("torch")
    B.build()
    assert os.path.exists(B.LIB) and os.path.exists(B.BINDING) and no_compiler[-1][0] == "g++"


@pytest.mark.parametrize("missing", ["torch", "headers"])
def test_without(missing, no_compiler, monkeypatch, tmp_path, capsys):
    with open(B.BINDING, "w"):
        pass  # of an earlier build: it would not fit the library
    if missing == "torch":
        import builtins
        real = builtins.__import__

        def refuse(name, *a, **kw):
            if name == "torch":
                raise ImportError("No module named 'torch'")
            return real(name, *a, **kw)

        monkeypatch.setattr(builtins, "__import__", refuse)
    else:
        pytest.importorskip("torch")
        monkeypatch.setattr(sysconfig, "get_paths", lambda *a, **kw: {"include": str(tmp_path / "none")})
    assert B.build() == B.LIB
    assert os.path.exists(B.LIB) and not os.path.exists(B.BINDING)
    assert len(no_compiler) == 1 and "_gba_decode.so" in capsys.readouterr().out


def test_a_compiler_that_fails_is_an_error(no_compiler, monkeypatch):
    pytest.importorskip("torch")
    run = B.subprocess.run

    def fail(cmd, **kw):
        if cmd[0] == "g++":
            raise B.subprocess.CalledProcessError(1, cmd)
        return run(cmd, **kw)

    monkeypatch.setattr(B.subprocess, "run", fail)
    with pytest.raises(B.subprocess.CalledProcessError):
        B.build()
