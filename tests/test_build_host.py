"""What a build makes where a part of the toolchain is missing, on small sources of
its own in another folder."""
import os

import pytest

from paper_2504_13850_gb300 import build


@pytest.fixture
def sources(tmp_path, monkeypatch):
    csrc = tmp_path / "csrc"
    csrc.mkdir()
    (csrc / "one.cu").write_text('extern "C" int one() { return 1; }\n')
    (csrc / "fo_binding.cpp").write_text('extern "C" int two() { return 2; }\n')
    for name, value in (("CSRC", csrc), ("BUILD", tmp_path / "_build"), ("OUT", tmp_path / "libfedoptima.so"), ("BINDING", tmp_path / "_binding.so")):
        monkeypatch.setattr(build, name, str(value))
    monkeypatch.setattr(build, "SOURCES", ["one.cu"])
    return csrc


@pytest.mark.parametrize("missing", ["torch", "headers", "g++"])
def test_the_library_needs_no_torch_and_no_compiler_but_nvcc(sources, monkeypatch, capfd, tmp_path, missing):
    if missing == "torch":
        find = build.importlib.util.find_spec
        monkeypatch.setattr(build.importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    elif missing == "headers":
        monkeypatch.setattr(build, "_torch", lambda: str(tmp_path))
    else:
        which = build.shutil.which
        monkeypatch.setattr(build.shutil, "which", lambda name, *a, **kw: None if name == "g++" else which(name, *a, **kw))
    with open(build.BINDING, "w") as f:
        f.write("made for another torch")
    assert build.build() == build.OUT and os.path.exists(build.OUT)
    assert not os.path.exists(build.BINDING) and "_binding.so is left out" in capfd.readouterr().err


def test_a_binding_that_does_not_compile_raises_behind_the_library(sources):
    (sources / "fo_binding.cpp").write_text("#error not this one\n")
    with pytest.raises(RuntimeError, match="not this one"):
        build.build()
    assert os.path.exists(build.OUT)


def test_another_torch_gets_another_binding(sources, monkeypatch, tmp_path):
    """Whatever the dates of its files."""
    os.makedirs(build.BUILD)
    root = tmp_path / "torch"
    (root / "include").mkdir(parents=True)
    monkeypatch.setattr(build, "_torch", lambda: str(root))
    said = []
    run = build._run
    monkeypatch.setattr(build, "_run", lambda *a: said.append(a[1]) or run(*a))
    for version, compiled in (("2.9.1", 1), ("2.9.1", 1), ("2.11.0", 2), ("2.11.0", 2), ("2.9.1", 3)):
        (root / "version.py").write_text(f"__version__ = '{version}'\n")
        os.utime(root / "version.py", (0, 0))
        build._compile_binding()
        assert len(said) == compiled
