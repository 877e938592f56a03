"""The in-tree build: the C library does not depend on the torch module, and that module follows the torch it was built for."""
import os
import subprocess

import pytest

from paper_2409_15104_b200 import build


@pytest.fixture
def fake(monkeypatch, tmp_path):
    """The build with its outputs in a folder of its own and commands that only write their output file."""
    ran = []

    def run(cmd, check):
        out = cmd[cmd.index("-o") + 1]
        ran.append(os.path.basename(out))
        if os.path.basename(cmd[0]) == "no-such-compiler":
            raise subprocess.CalledProcessError(1, cmd)
        open(out, "w").close()

    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libpec.so"))
    monkeypatch.setattr(build, "TORCH_MODULE", str(tmp_path / "_pec_torch.so"))
    return ran


def test_the_c_library_is_built_where_the_torch_module_cannot_be(fake, monkeypatch):
    monkeypatch.setenv("CXX", "no-such-compiler")
    with pytest.raises(subprocess.CalledProcessError):
        build.build(force=True)
    assert fake == ["libpec.so", "_pec_torch.so"] and os.path.exists(build.LIB)


def test_nothing_is_rebuilt_without_a_reason(fake):
    build.build()
    build.build()
    assert sorted(fake) == ["_pec_torch.so", "libpec.so"]


@pytest.mark.parametrize("other", ["torch", "python"])
def test_the_torch_module_is_rebuilt_for_another_torch_or_python(fake, monkeypatch, other):
    import sys
    import torch
    build.build()
    del fake[:]
    if other == "torch":
        monkeypatch.setattr(torch, "__version__", "0.0.1")
    else:
        monkeypatch.setattr(sys, "version", "0.0.1")
    build.build()
    assert fake == ["_pec_torch.so"]
    build.build()
    assert fake == ["_pec_torch.so"]
