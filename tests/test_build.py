"""What building the library needs (no compiler runs here)."""
import os
import subprocess

import pytest

from paper_2406_13170_b200 import build as amph_build


@pytest.fixture
def commands(monkeypatch, tmp_path):
    """The commands that a build runs, with targets in a place of their own; "fail": those that cannot be started or return an error."""
    seen = {"ran": [], "fail": {}}
    monkeypatch.setattr(amph_build, "LIB", str(tmp_path / "libamph.so"))
    monkeypatch.setattr(amph_build, "OPS", str(tmp_path / "torch_ops.so"))

    def made(cmd):
        target = os.path.basename(cmd[cmd.index("-o") + 1])
        seen["ran"].append(target)
        how = seen["fail"].get(target)
        if isinstance(how, Exception):
            raise how
        if not how:
            open(cmd[cmd.index("-o") + 1], "w").close()
        return how or 0

    class Popen:
        def __init__(self, cmd):
            self.args, self.rc = cmd, made(cmd)

        def wait(self):
            return self.rc

    def run(cmd, check):
        rc = made(cmd)
        if rc:
            raise subprocess.CalledProcessError(rc, cmd)

    monkeypatch.setattr(amph_build.subprocess, "Popen", Popen)
    monkeypatch.setattr(amph_build.subprocess, "run", run)
    return seen


def test_both_are_built_once(commands):
    assert amph_build.build() == amph_build.LIB
    assert sorted(commands["ran"]) == ["libamph.so", "torch_ops.so"]
    amph_build.build()
    assert len(commands["ran"]) == 2
    amph_build.build(force=True)
    assert len(commands["ran"]) == 4


@pytest.mark.parametrize("fault", [FileNotFoundError("g++"), 1], ids=["no_compiler", "no_headers"])
def test_the_library_needs_no_torch_headers(commands, fault):
    commands["fail"]["torch_ops.so"] = fault
    with pytest.raises(RuntimeError, match="torch_ops.so was not built"):
        amph_build.build()
    assert os.path.exists(amph_build.LIB) and not os.path.exists(amph_build.OPS)
    assert amph_build.build(ops=False) == amph_build.LIB
    assert commands["ran"] == ["torch_ops.so", "libamph.so"]              # the library is not built again


@pytest.mark.parametrize("fault", [ImportError("torch"), RuntimeError("torch of another CUDA")], ids=["no_torch", "another_torch"])
def test_without_torch(commands, monkeypatch, fault):
    def command():
        raise fault
    monkeypatch.setattr(amph_build, "_ops_command", command)
    with pytest.raises(RuntimeError, match="torch"):
        amph_build.build()
    assert os.path.exists(amph_build.LIB)


def test_a_library_that_does_not_compile(commands):
    commands["fail"]["libamph.so"] = 2
    with pytest.raises(subprocess.CalledProcessError):
        amph_build.build()
