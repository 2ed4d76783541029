"""How the compiled parts are built and loaded: the library by itself, the binding's C++ part at its first call."""
import os
import sysconfig

import pytest
import torch

from paper_2410_05076_b200 import binding, build


@pytest.fixture()
def unloaded(monkeypatch):
    binding.load()                                        # the library is built
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.setattr(binding, "_fast", None)


def broken(*args, **kw):
    raise OSError("no compiler for C++20")


def test_the_library_loads_where_the_cpp_part_cannot_be_built(unloaded, monkeypatch, tmp_path):
    monkeypatch.setattr(build, "fast_path", lambda: str(tmp_path / "_fast_call-missing.so"))
    monkeypatch.setattr(build, "build_fast", broken)
    assert binding.load().tidal_strerror
    td = binding.Tidal.__new__(binding.Tidal)
    td.lib, td.ctx, td.device = binding.load(), binding.C.c_void_p(), 0
    for _ in range(2):                                    # and what failed is named, every time
        with pytest.raises(ImportError, match="_fast_call-missing.so.*no compiler"):
            td.kv_write(binding.tidal_kv_t(), None, None, None)


def test_the_cpp_part_loads_at_its_first_call(unloaded):
    binding.load()
    assert binding._fast is None
    td = binding.Tidal.__new__(binding.Tidal)
    td.lib, td.ctx, td.device = binding.load(), binding.C.c_void_p(), 0
    with pytest.raises(ValueError, match="slots"):
        td.kv_write(binding.tidal_kv_t(), None, None, None)
    assert binding._fast is not None


def test_the_cpp_part_of_another_python_or_torch_is_not_taken(monkeypatch):
    path = build.fast_path()
    assert os.path.dirname(path) == os.path.dirname(build.LIB)
    assert torch.__version__ in path and path.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert build.fast_path() != path and build.fast_is_stale()


def test_the_message_names_the_library_that_failed(unloaded, monkeypatch, tmp_path):
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libtidal.so"))
    monkeypatch.setattr(build, "build", broken)
    with pytest.raises(ImportError, match="libtidal.so is missing"):
        binding.load()
