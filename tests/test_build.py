"""The build: what is linked when, and what it is compiled against.  A one-function source stands for the library."""
import os

import pytest

from paper_2607_14557_gb300 import build


@pytest.fixture
def small(tmp_path, monkeypatch):
    (tmp_path / "one.cu").write_text('extern "C" int one() { return 1; }\n')
    (tmp_path / "binding.cpp").write_text("// nothing\n")
    for name, value in dict(CSRC=str(tmp_path), BUILD=str(tmp_path / "b"), LIB=str(tmp_path / "libseer.so"), BINDING=str(tmp_path / "_seer_binding.so"),
                            SOURCES=["one.cu"], HEADERS=[]).items():
        monkeypatch.setattr(build, name, value)
    return tmp_path


def test_the_library_is_there_where_the_binding_cannot_be_compiled(small, monkeypatch):
    def refuse(nv):
        raise RuntimeError("no Python.h")

    monkeypatch.setattr(build, "_compile_binding", refuse)
    with pytest.raises(RuntimeError, match="Python.h"):
        build.build()
    assert os.path.exists(build.LIB)
    before = os.stat(build.LIB).st_mtime_ns
    with pytest.raises(RuntimeError, match="Python.h"):     # the library is not compiled again for that
        build.build()
    assert os.stat(build.LIB).st_mtime_ns == before


def test_another_torch_or_python_compiles_the_binding_again(small, monkeypatch):
    done = []
    monkeypatch.setattr(build, "_compile_binding", lambda nv: str(small / "binding.cpp"))

    def run(cmd, what):
        done.append(what)
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(build, "_run", run)
    open(build.LIB, "w").close()
    build.build()
    assert done == ["linking the binding"]
    build.build()
    assert done == ["linking the binding"]
    monkeypatch.setattr(build, "_binding_for", lambda: "another torch")
    build.build()
    assert done == ["linking the binding"] * 2
