"""What the build makes of what: the C library by itself, the marshalling module for one torch and one Python."""
import os

import pytest


@pytest.fixture
def b(tmp_path, monkeypatch):
    """The package's build, of one small source, into a folder of its own."""
    from paper_2205_01435_gb300 import _build
    src = tmp_path / "one.cu"
    src.write_text('extern "C" int one() { return 1; }\n')
    ext = tmp_path / "ext.cpp"
    ext.write_text('extern "C" int two() { return 2; }\n')
    for name, at in (("LIB", "libone.so"), ("EXT", "_ext.so"), ("BUILD", "objects")):
        monkeypatch.setattr(_build, name, str(tmp_path / at))
    monkeypatch.setattr(_build, "EXT_SRC", str(ext))
    monkeypatch.setattr(_build, "_sources", lambda: [str(src)])
    return _build


def test_the_library_is_built_without_the_module(b, recwarn):
    """Where the marshalling module does not compile (no torch, no Python headers) the C library is there all the same, and
    no older module stays beside it."""
    with open(b.EXT_SRC, "w") as f:
        f.write("#error no headers\n")
    with open(b.EXT, "w") as f:
        f.write("older")
    assert b.build(force=True) == b.LIB
    assert os.path.exists(b.LIB) and not os.path.exists(b.EXT)
    assert any("no headers" in str(w.message) for w in recwarn.list)
    assert not b.up_to_date()
    built = os.path.getmtime(b.LIB)
    b.build()  # (the module is tried again, the library is not made again)
    assert os.path.getmtime(b.LIB) == built


def test_the_module_is_built_for_one_torch(b, monkeypatch):
    b.build()
    assert b.up_to_date()
    made = os.path.getmtime(b.LIB), os.path.getmtime(b.EXT)
    version = b.importlib.metadata.version
    monkeypatch.setattr(b.importlib.metadata, "version", lambda name: version(name) + ".other")
    assert not b.up_to_date()
    b.build()
    assert b.up_to_date() and os.path.getmtime(b.LIB) == made[0] and os.path.getmtime(b.EXT) > made[1]
