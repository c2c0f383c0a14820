"""The build's parts: the integer library does not hang on the compiled calls of the microscaled operators, whose module
belongs to one interpreter."""
import os
import sysconfig

import pytest

import paper_2603_04359_gb300 as cat
from fake_runtime import ensure_built
from paper_2603_04359_gb300 import build as catbuild


def test_library_is_linked_where_the_calls_do_not_compile(tmp_path, monkeypatch):
    """Without torch's C++ headers, say: the build fails and says why, with the library in place."""
    lib = str(tmp_path / "libcatw4a4.so")
    monkeypatch.setattr(catbuild, "LIB", lib)
    monkeypatch.setattr(catbuild, "BUILD", str(tmp_path / "objects"))
    monkeypatch.setattr(catbuild, "_compile", lambda src, verbose: src)

    def link(cmd, what):
        open(cmd[cmd.index("-o") + 1], "w").close()

    def no_headers():
        raise RuntimeError("compiling mx_calls.cpp failed:\nATen/core/Tensor.h: No such file or directory")
    monkeypatch.setattr(catbuild, "_run", link)
    monkeypatch.setattr(catbuild, "_compile_calls", no_headers)
    with pytest.raises(RuntimeError, match="mx_calls.cpp"):
        catbuild.build()
    assert os.path.exists(lib)


def test_module_of_the_calls_is_one_interpreters():
    """Another interpreter does not find it (and says so), instead of loading it and failing inside."""
    ensure_built()
    assert os.path.basename(catbuild.CALLS) == "_mx_calls" + sysconfig.get_config_var("EXT_SUFFIX")
    assert os.path.samefile(cat._calls().__file__, catbuild.CALLS)
