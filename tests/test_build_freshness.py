"""When a build counts as fresh, and what a failed one leaves behind (host only: compilers are stand-ins)."""
import os
import subprocess
import sysconfig

import pytest

from paper_2512_21835_gb300 import build as B


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """An empty package folder with one source file of each kind."""
    csrc = tmp_path / "csrc"
    csrc.mkdir()
    for f in ("a.cu", "calls.c"):
        (csrc / f).write_text("")
    monkeypatch.setattr(B, "HERE", str(tmp_path))
    monkeypatch.setattr(B, "CSRC", str(csrc))
    monkeypatch.setattr(B, "OUT", str(tmp_path / "libloip.so"))
    monkeypatch.setattr(B, "CALLS", str(tmp_path / os.path.basename(B.CALLS)))
    monkeypatch.setattr(B, "BUILD", str(tmp_path / "_build"))
    monkeypatch.setattr(B, "SOURCES", ["a.cu"])
    monkeypatch.setattr(B, "_nvcc", lambda: "nvcc")
    return tmp_path


def compiler(monkeypatch, fails=""):
    """Every command writes its output file, except one that names `fails`; returns the commands."""
    commands = []

    def run(cmd, **kw):
        commands.append(cmd)
        bad = bool(fails) and any(fails in c for c in cmd)
        if not bad:
            with open(cmd[cmd.index("-o") + 1], "w") as f:
                f.write(" ".join(cmd))
        return subprocess.CompletedProcess(cmd, int(bad), "", "no such header" if bad else "")

    monkeypatch.setattr(B.subprocess, "run", run)
    return commands


def age(path, t):
    os.utime(path, (t, t))


def test_a_failed_extension_leaves_the_build_stale(tree, monkeypatch):
    compiler(monkeypatch)
    B.build()
    assert not B._stale()
    for f, t in ((B.OUT, 1100), (B.CALLS, 1100), (tree / "csrc" / "a.cu", 1000), (tree / "csrc" / "calls.c", 1200)):
        age(f, t)
    assert B._stale()
    compiler(monkeypatch, fails="calls.c")
    for _ in range(2):  # the second build fails too, and does not find the first one's library fresh
        with pytest.raises(RuntimeError, match="calls.c"):
            B.build()
        assert B._stale()


def test_both_files_are_newer_than_every_source(tree, monkeypatch):
    compiler(monkeypatch)
    B.build()
    for f in (tree / "csrc" / "a.cu", tree / "csrc" / "calls.c"):
        age(f, 1000)
    for old, new in ((B.CALLS, B.OUT), (B.OUT, B.CALLS)):
        age(old, 900)
        age(new, 1100)
        assert B._stale()
    age(B.CALLS, 1100)
    age(B.OUT, 1100)
    assert not B._stale()


def test_the_extension_is_of_this_interpreter():
    assert os.path.basename(B.CALLS) == "_calls" + sysconfig.get_config_var("EXT_SUFFIX")


def test_one_compiler(tree, monkeypatch):
    """Everything goes through nvcc, which finds the host's compiler."""
    commands = compiler(monkeypatch)
    B.build()
    assert {c[0] for c in commands} == {"nvcc"}


def test_without_python_headers(tree, monkeypatch):
    """The library is built all the same, and no module of an earlier build stays beside it."""
    commands = compiler(monkeypatch)
    B.build()
    monkeypatch.setattr(B.sysconfig, "get_paths", lambda: dict(include=str(tree / "nowhere")))
    os.utime(tree / "csrc" / "a.cu", (os.path.getmtime(B.OUT) + 10,) * 2)
    commands.clear()
    B.build()
    assert commands and not any("calls.c" in c for cmd in commands for c in cmd)
    assert os.path.exists(B.OUT) and not os.path.exists(B.CALLS)
    age(tree / "csrc" / "a.cu", 1000)
    age(tree / "csrc" / "calls.c", 1000)
    assert not B._stale()


def test_entries_without_the_extension(monkeypatch):
    """Without it the windowed-serving entries are called through ctypes, with the same refusals."""
    import ctypes as C

    from paper_2512_21835_gb300 import loip
    B.build()
    monkeypatch.setattr(B, "CALLS", B.CALLS + ".missing")
    monkeypatch.setattr(loip, "_lib", None)
    L = loip.lib()
    for name in ("loip_k_qk_append", "loip_k_window_attention_q8", "loip_k_cache_read_q8"):
        sig = loip._SIGS[name][1]
        zero = [0.0 if t is C.c_float else None if t is C.c_void_p else 0 for t in sig]
        assert isinstance(getattr(L, name), C._CFuncPtr) and getattr(L, name)(*zero) == loip.ERR_INVALID
