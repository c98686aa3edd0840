"""What is built when: the library before the binding and without it, the binding again when torch or Python change."""
import os
import subprocess

import pytest


@pytest.fixture
def build(monkeypatch, tmp_path):
    """The build module writing under tmp_path, with compilers that only note the command and write their output file."""
    from paper_2607_17644_b200 import build as module
    for name in ("LIB_PATH", "DEBUG_LIB_PATH", "BINDING_PATH", "BINDING_STAMP"):
        monkeypatch.setattr(module, name, str(tmp_path / os.path.basename(getattr(module, name))))
    module.ran = []

    def compiler(cmd, check):
        assert check
        module.ran.append(os.path.basename(cmd[0]))
        if cmd[0] in module.missing:
            raise FileNotFoundError(cmd[0])
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("built")

    module.missing = ()
    monkeypatch.setattr(subprocess, "run", compiler)
    yield module
    del module.ran, module.missing


def test_library_does_not_need_the_binding(build):
    build.missing = ("g++",)
    with pytest.raises(FileNotFoundError):
        build.build()
    assert os.path.exists(build.LIB_PATH) and build.ran == ["nvcc", "g++"]
    assert build.build_library() == build.LIB_PATH and build.ran == ["nvcc", "g++"]


def test_binding_follows_torch_and_python(build, monkeypatch):
    build.build()
    assert build.ran == ["nvcc", "g++"] and os.path.exists(build.BINDING_PATH)
    build.build()
    assert build.ran == ["nvcc", "g++"]                              # nothing changed
    monkeypatch.setattr(build.importlib.metadata, "version", lambda name: "1.2.3")
    build.build()
    build.build()
    assert build.ran == ["nvcc", "g++", "g++"]
    os.remove(build.BINDING_STAMP)                                   # not known what it was built with
    build.build()
    assert build.ran == ["nvcc", "g++", "g++", "g++"]
    build.build(force=True, debug=True)
    assert build.ran[4:] == ["nvcc", "g++"] and os.path.exists(build.DEBUG_LIB_PATH)
