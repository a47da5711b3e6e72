"""The binding's compiled checks are an addition: the library builds and loads without them, and a build of them for another Python or torch is
not loaded."""
import os
import time
import warnings

import pytest
import torch

from paper_2608_20375_b200 import binding, build


@pytest.fixture
def no_compiler(monkeypatch, tmp_path):
    """Nothing on the path, and compiled checks that are older than their source; the CUDA library is there."""
    build.build()
    newer = tmp_path / "marshal.cpp"
    newer.write_text("")
    os.utime(newer, (time.time() + 1000,) * 2)
    monkeypatch.setattr(build, "_marshal_deps", lambda: [str(newer)])
    monkeypatch.setenv("PATH", str(tmp_path))


@pytest.fixture
def unloaded(monkeypatch):
    for name in ("_lib", "_fast"):
        monkeypatch.setattr(binding, name, None)


def test_the_library_builds_without_a_host_compiler(no_compiler):
    assert not build.needs_build()
    with pytest.warns(UserWarning, match="compiled checks"):
        assert build.build() == build.LIB


def test_the_library_loads_without_a_host_compiler(no_compiler, unloaded):
    with pytest.warns(UserWarning, match="compiled checks"):
        lib = binding.load_library()
    assert lib.graft_version() and binding._fast is None


def test_checks_that_do_not_compile(monkeypatch, tmp_path, unloaded):
    build.build()
    broken = tmp_path / "marshal.cpp"
    broken.write_text("#error\n")
    os.utime(broken, (time.time() + 1000,) * 2)
    command = build._marshal_command
    monkeypatch.setattr(build, "_marshal_deps", lambda: [str(broken)])
    monkeypatch.setattr(build, "_marshal_command", lambda *a: [str(broken) if x.endswith("marshal.cpp") else x for x in command(*a)])
    with pytest.warns(UserWarning, match="compiled checks"):
        binding.load_library()
    assert binding._fast is None


@pytest.mark.parametrize("what", ["torch", "python"])
def test_checks_for_another_torch_or_python_are_not_loaded(what, monkeypatch, tmp_path, unloaded):
    build.build()
    monkeypatch.setenv("PATH", str(tmp_path))
    if what == "torch":
        monkeypatch.setattr(torch, "__version__", "1.0.0+other")
    else:
        monkeypatch.setattr(build.sysconfig, "get_config_var", lambda name: ".cpython-399-x86_64-linux-gnu.so")
    with pytest.warns(UserWarning, match="compiled checks"):
        binding.load_library()
    assert binding._fast is None


def test_checks_that_are_there_are_loaded(unloaded):
    build.build()
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        binding.load_library()
    assert binding._fast is not None
