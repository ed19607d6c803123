"""What the build asks of a machine."""
import os
import subprocess

import pytest

from paper_2101_09808_amd import build


@pytest.fixture()
def commands(tmp_path, monkeypatch):
    """The commands that a build runs, in a folder of their own: hipcc's outputs
    appear, every other program is missing."""
    ran = []

    def run(cmd, **kw):
        ran.append(cmd)
        if cmd[0] != build.HIPCC:
            raise FileNotFoundError(2, "No such file or directory", cmd[0])
        open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(build, "OBJ", str(tmp_path / "obj"))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libconvfwd.so"))
    monkeypatch.setattr(build, "SEQ", str(tmp_path / "_seq.so"))
    monkeypatch.setattr(build.subprocess, "run", run)
    return ran


def test_the_library_needs_hipcc_alone(commands):
    assert build.build_library() == build.LIB and os.path.exists(build.LIB)
    assert {c[0] for c in commands} == {build.HIPCC} and len(commands) == len(build.SOURCES) + 1


def test_a_module_that_cannot_be_built_leaves_the_library_and_says_so(commands):
    with pytest.raises(RuntimeError, match="is built, the Python module is not.*g\\+\\+"):
        build.build()
    assert os.path.exists(build.LIB) and not os.path.exists(build.SEQ)
