"""What the build makes of a machine that can compile the library but not the Python binding."""
import os

import pytest

from paper_2601_11553_b200 import build


def test_the_library_is_built_without_a_compiler_for_the_binding(tmp_path, monkeypatch, capfd):
    build.build()
    monkeypatch.setattr(build, "BINDING_PATH", str(tmp_path / "_ops_binding.so"))
    monkeypatch.setenv("CXX", str(tmp_path / "no-such-compiler"))
    before = os.path.getmtime(build.LIB_PATH)
    assert build.build() == build.LIB_PATH
    assert os.path.getmtime(build.LIB_PATH) == before               # which was up to date
    assert not os.path.exists(build.BINDING_PATH)
    assert "ops_binding.cpp" in capfd.readouterr().err
    with pytest.raises(RuntimeError, match="ops_binding.cpp"):
        build.build_binding()


def test_an_outdated_binding_is_not_left_beside_a_new_library(tmp_path, monkeypatch):
    lib, binding = tmp_path / "libpercache.so", tmp_path / "_ops_binding.so"
    binding.write_text("old")
    os.utime(binding, (1, 1))
    monkeypatch.setattr(build, "LIB_PATH", str(lib))
    monkeypatch.setattr(build, "BINDING_PATH", str(binding))
    monkeypatch.setattr(build, "build_library", lambda verbose=False: lib.write_text("new"))
    monkeypatch.setenv("CXX", str(tmp_path / "no-such-compiler"))
    assert build.build() == str(lib)
    assert lib.exists() and not binding.exists()
