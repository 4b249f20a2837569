"""The binding's host half belongs to the library it was built beside and to the torch it was built against."""
import os
import types

import pytest
import torch

from paper_2606_12950_amd import _train, build


def test_another_torch_is_refused(monkeypatch):
    _train.load()
    monkeypatch.setattr(_train, "_lib", None)
    monkeypatch.setattr(torch, "__version__", "1.2.3+other")
    with pytest.raises(RuntimeError, match=r"1\.2\.3\+other.*build"):
        _train.load()
    monkeypatch.undo()
    _train.load()


def test_a_failed_build_installs_nothing(monkeypatch, tmp_path):
    """Whichever part fails, the libraries that are there stay, all of them."""
    libs = [str(tmp_path / n) for n in ("a.so", "b.so", "c.so")]
    for name, lib in zip(("LIB", "CALIBRATE_LIB", "TENSORS_LIB"), libs):
        monkeypatch.setattr(build, name, lib)
        open(lib, "w").write("old")

    def link(cmd, **kw):
        open(cmd[cmd.index("-o") + 1], "w").write("new")
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")

    def host_half(outdir, verbose):
        raise RuntimeError("no host compiler")

    monkeypatch.setattr(build, "_compile", lambda src, outdir, verbose: os.path.join(outdir, src))
    monkeypatch.setattr(build, "_compile_tensors", host_half)
    monkeypatch.setattr(build.subprocess, "run", link)
    monkeypatch.setattr(build, "HIPCC", os.devnull)
    with pytest.raises(RuntimeError, match="no host compiler"):
        build.build()
    assert [open(lib).read() for lib in libs] == ["old"] * 3
