"""What the build does when its parts are missing or out of date (nothing is compiled here)."""
import os

import pytest
import torch

import paper_2604_05438_b200.binding as B
import paper_2604_05438_b200.build as build


@pytest.fixture
def built(tmp_path, monkeypatch):
    """A library and a module of the paged calls that are up to date, somewhere else."""
    for name in ("LIB", "BINDING"):
        path = tmp_path / os.path.basename(getattr(build, name))
        path.write_bytes(b"built")
        monkeypatch.setattr(build, name, str(path))
    return tmp_path


def _no_compiler(*a, **k):
    raise AssertionError("nothing is to be compiled")


def test_what_is_up_to_date_is_left_alone(built, monkeypatch):
    monkeypatch.setattr(build.subprocess, "run", _no_compiler)
    assert not build.needs_build()
    assert build.build_library() == build.LIB


def test_a_library_does_not_need_the_module(built, monkeypatch):
    # no C++ compiler: the library is there all the same, and no old module is left beside it
    monkeypatch.setenv("CXX", "/nonexistent/c++")
    for old in (True, False):
        if old:
            os.utime(build.BINDING, (1, 1))
        with pytest.warns(UserWarning, match="paged"):
            assert build.build_library() == build.LIB
        assert not os.path.exists(build.BINDING)
        assert open(build.LIB, "rb").read() == b"built"


def test_a_module_that_does_not_compile_is_an_error_of_its_own_build(built, monkeypatch):
    monkeypatch.setenv("CXX", "false")
    with pytest.raises(RuntimeError, match="_paged_binding"):
        build.build_binding()


def test_another_torch_makes_the_module_out_of_date(built, tmp_path, monkeypatch):
    (tmp_path / "version.py").write_text("")
    monkeypatch.setattr(build, "_torch_root", lambda: str(tmp_path))
    t = os.path.getmtime(build.BINDING)
    os.utime(tmp_path / "version.py", (t - 5, t - 5))
    assert not build.binding_needs_build()
    os.utime(tmp_path / "version.py", (t + 5, t + 5))
    assert build.binding_needs_build() and not build.library_needs_build()


def test_a_module_of_another_torch_is_refused(monkeypatch):
    build.build_library()
    assert B._native().torch_version == torch.__version__
    monkeypatch.setattr(B, "_native_module", None)
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    with pytest.raises(RuntimeError, match="0.0.1"):
        B._native()
