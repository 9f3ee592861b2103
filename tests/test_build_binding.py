"""The build of the module of the calls on rows: the library does not depend on it, and a module of another interpreter or torch
is built anew instead of being loaded."""
import os

import pytest

from paper_2608_13255_gb300 import build as gbuild


@pytest.fixture
def gc(monkeypatch):
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    monkeypatch.setattr(geocache, "_ROWS", None)
    return geocache


def _elsewhere(monkeypatch, tmp_path):
    """A build of one empty kernel into a folder of its own."""
    for name in ("LIB", "BINDING", "BINDING_FOR"):
        monkeypatch.setattr(gbuild, name, str(tmp_path / os.path.basename(getattr(gbuild, name))))
    monkeypatch.setattr(gbuild, "LIBDIR", str(tmp_path))
    src = tmp_path / "tiny.cu"
    src.write_text('__global__ void tiny() {}\nextern "C" int tiny_version(void) { return 1; }\n')
    monkeypatch.setattr(gbuild, "_sources", lambda: [str(src)])


def test_a_module_of_another_torch_is_stale(gc, monkeypatch, tmp_path):
    assert not gbuild.is_stale() and gbuild.binding_was_for() == gbuild.binding_for()
    monkeypatch.setattr(gbuild, "BINDING_FOR", str(tmp_path / "for"))
    for text in (None, "cpython-39, torch 1.0"):
        if text:
            (tmp_path / "for").write_text(text)
        assert gbuild.binding_is_stale() and gbuild.is_stale() and not gbuild.library_is_stale()
        with pytest.raises(RuntimeError, match="was built for"):
            gc._rows_binding()


def test_the_library_alone(gc, monkeypatch, tmp_path, capfd):
    monkeypatch.setattr(gbuild, "binding_needs", lambda: "Python.h")
    with monkeypatch.context() as m:
        _elsewhere(m, tmp_path)
        assert gbuild.build() == gbuild.LIB and os.path.exists(gbuild.LIB) and not os.path.exists(gbuild.BINDING)
        assert "it needs Python.h" in capfd.readouterr().err
        assert not gbuild.is_stale()  # what cannot be built here is not waited for
        with pytest.raises(RuntimeError, match="needs Python.h"):
            gc._rows_binding()


def test_a_module_that_does_not_compile(gc, monkeypatch, tmp_path, capfd):
    _elsewhere(monkeypatch, tmp_path)
    bad = tmp_path / "bad.cpp"
    bad.write_text("this is no C++\n")
    monkeypatch.setattr(gbuild, "_binding_source", lambda: str(bad))
    with pytest.raises(RuntimeError, match="bad.cpp"):
        gbuild.build()
    assert os.path.exists(gbuild.LIB) and not os.path.exists(gbuild.BINDING)
    assert gbuild.is_stale() and not gbuild.library_is_stale()
