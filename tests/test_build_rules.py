"""When the build makes the head's extension anew (no GPU, no compiler: its commands are replaced)."""
import importlib.metadata
import os

import pytest

from paper_2604_01000_b200 import build


@pytest.fixture
def made(tmp_path, monkeypatch):
    """The build in an empty folder, without CUDA sources; returns the list of the extension's links so far."""
    links, real = [], build.subprocess.run
    for name in ("LIB", "LIB_DEBUG"):
        path = tmp_path / (name + ".so")
        path.write_bytes(b"")
        monkeypatch.setattr(build, name, str(path))
    monkeypatch.setattr(build, "OBJ", str(tmp_path / "obj"))
    monkeypatch.setattr(build, "OBJ_DEBUG", str(tmp_path / "obj_debug"))
    monkeypatch.setattr(build, "HEAD", str(tmp_path / "_head.so"))
    monkeypatch.setattr(build, "sources", lambda: [])
    monkeypatch.setattr(build, "head_commands", lambda: (["true"], ["touch"]))

    def run(cmd, **kw):
        assert cmd[0] in ("true", "touch"), cmd
        links.extend(cmd[1:2])
        return real(cmd, **kw)
    monkeypatch.setattr(build.subprocess, "run", run)
    return links


@pytest.mark.parametrize("debug", [False, True])
def test_either_build_makes_the_extension_once(made, debug):
    build.build(debug=debug)
    assert os.path.exists(build.HEAD) and len(made) == 1
    build.build(debug=debug)
    build.build(debug=not debug)
    assert len(made) == 1


def test_another_torch_or_python_makes_it_anew(made, monkeypatch):
    build.build()
    version = importlib.metadata.version("torch")
    monkeypatch.setattr(importlib.metadata, "version", lambda name: version + ".1" if name == "torch" else "")
    build.build()
    assert len(made) == 2
    monkeypatch.setattr(build.sysconfig, "get_config_var", lambda name: "cpython-999" if name == "SOABI" else None)
    build.build()
    build.build()
    assert len(made) == 3


def test_a_link_that_fails_leaves_no_mark_of_success(made, monkeypatch):
    monkeypatch.setattr(build, "head_commands", lambda: (["true"], ["touch", "/nonexistent/x"]))
    with pytest.raises(RuntimeError):
        build.build()
    monkeypatch.setattr(build, "head_commands", lambda: (["true"], ["touch"]))
    build.build()
    assert os.path.exists(build.HEAD)
