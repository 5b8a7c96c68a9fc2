"""The library builds by itself; what the argument marshaller needs besides is asked for by its own wrappers alone."""
import os
import subprocess

import pytest

from paper_2407_14057_b200 import binding, build


@pytest.mark.parametrize("error", [ImportError("no torch"), FileNotFoundError("no compiler"),
                                   subprocess.CalledProcessError(1, "g++")])
def test_library_without_the_marshaller(error, monkeypatch, capfd):
    build.build()   # up to date from here on

    def fails(force=False):
        raise error

    monkeypatch.setattr(build, "build_call", fails)
    assert build.build() == build.LIB and os.path.exists(build.LIB)
    assert "lazycall.so was not built" in capfd.readouterr().err
    assert binding.lib().lazy_keep_count(100, 5000, 100) == 50


def test_wrappers_say_that_the_marshaller_is_missing(monkeypatch, tmp_path):
    build.build()
    monkeypatch.setattr(binding, "CALL_PATH", str(tmp_path / "lazycall.so"))
    monkeypatch.setattr(binding, "_call", None)
    with pytest.raises(RuntimeError, match="is missing"):
        binding._native()


def test_a_marshaller_that_cannot_be_made_anew_is_gone(monkeypatch, tmp_path):
    """An old one could expect other entry points than the library has."""
    old = tmp_path / "lazycall.so"
    old.write_bytes(b"old")
    monkeypatch.setattr(build, "CALL_LIB", str(old))
    monkeypatch.setattr(build, "CALL_STAMP", str(tmp_path / "stamp.txt"))
    monkeypatch.setenv("CXX", "false")
    with pytest.raises(subprocess.CalledProcessError):
        build.build_call()
    assert not old.exists()
