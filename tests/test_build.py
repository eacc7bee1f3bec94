"""What build.py builds when.  The commands are recorded, not run."""
import pytest

from paper_2107_13490_b200 import build


@pytest.fixture
def commands(monkeypatch, tmp_path):
    """The commands that a build would run; each leaves its output file behind."""
    ran = []

    def run(cmd, check):
        ran.append(cmd[0])
        with open(cmd[cmd.index("-o") + 1], "w"):
            pass

    monkeypatch.setattr(build.subprocess, "run", run)
    for name in ("LIB", "CHECK_LIB", "CALLS"):
        monkeypatch.setattr(build, name, str(tmp_path / name))
    monkeypatch.setenv("NVCC", "nvcc")
    return ran


def test_library_and_extension_are_built_once(commands):
    build.build()
    assert commands == ["nvcc", "g++"]
    build.build()
    assert commands == ["nvcc", "g++"]
    build.build(check=True)
    assert commands == ["nvcc", "g++", "nvcc"]


def test_the_library_needs_no_torch(commands, monkeypatch):
    monkeypatch.setattr(build, "torch_version", lambda: None)
    build.build()
    build.build(check=True)
    assert commands == ["nvcc", "nvcc"]


def test_the_library_alone(commands):
    build.build(calls=False)
    assert commands == ["nvcc"]


def test_the_extension_follows_torch(commands, monkeypatch):
    build.build_calls()
    build.build_calls()
    assert commands == ["g++"]
    monkeypatch.setattr(build, "torch_version", lambda: "another torch\n")
    build.build_calls()
    build.build_calls()
    assert commands == ["g++", "g++"]


def test_no_torch_is_no_version(monkeypatch):
    assert build.torch_version()

    def missing(name):
        raise build.importlib.metadata.PackageNotFoundError(name)

    monkeypatch.setattr(build.importlib.metadata, "version", missing)
    assert build.torch_version() is None
