"""The compiled binding is optional: where it does not compile, the library is built without it."""
import os
import sys

import pytest

from paper_2609_29219_gb300 import build as module


@pytest.fixture
def place(tmp_path, monkeypatch):
    """A binding of its own to build, with an older one there."""
    target = tmp_path / "_binding.so"
    target.write_bytes(b"older")
    monkeypatch.setattr(module, "BINDING", str(target))
    return target


def test_a_binding_that_does_not_compile_is_left_out(place, monkeypatch, capfd):
    tmp = str(place) + ".tmp"
    bad = [sys.executable, "-c", "import sys; print('no such member', file=sys.stderr); sys.exit(1)"]
    monkeypatch.setattr(module, "_binding_job", lambda force: (bad, tmp))
    assert module.build() == module.LIB and os.path.exists(module.LIB)
    assert not place.exists()  # the older one is of another source or torch
    err = capfd.readouterr().err
    assert "_binding.so" in err and "no such member" in err


def test_a_compiler_that_is_missing_too(place, monkeypatch, capfd):
    monkeypatch.setattr(module, "_binding_job", lambda force: (["/nonexistent/compiler"], str(place) + ".tmp"))
    assert module.build() == module.LIB
    assert not place.exists() and "_binding.so" in capfd.readouterr().err


def test_a_binding_that_compiles_is_put_in_place(place, monkeypatch):
    tmp = str(place) + ".tmp"
    good = [sys.executable, "-c", f"open({tmp!r}, 'wb').write(b'new')"]
    monkeypatch.setattr(module, "_binding_job", lambda force: (good, tmp))
    module.build()
    assert place.read_bytes() == b"new"
