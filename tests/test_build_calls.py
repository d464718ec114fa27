"""CPU: the library builds and its training calls work where the CPython callables cannot be built, and no interpreter gets another's."""
import itertools
import os
import shutil
import subprocess
import sys
import sysconfig

import pytest

from paper_2308_14352_b200 import binding as B
from paper_2308_14352_b200 import build
from tests.test_pycall import NAMES, _arguments


@pytest.fixture
def compilers(monkeypatch):
    """What build() would run."""
    ran = []
    monkeypatch.setattr(subprocess, "check_call", lambda cmd: ran.append(cmd))
    return ran


@pytest.mark.parametrize("what", ["g++", "Python.h"])
def test_the_library_is_built_without(compilers, monkeypatch, tmp_path, what):
    if what == "g++":
        monkeypatch.setattr(shutil, "which", lambda name: None)
    else:
        paths = dict(sysconfig.get_paths(), include=str(tmp_path))
        monkeypatch.setattr(sysconfig, "get_paths", lambda: paths)
    with pytest.warns(UserWarning, match=what.replace("+", r"\+")):
        assert build.build(force=True) == build.LIB_PATH
    assert [cmd[0] for cmd in compilers] == ["nvcc"]


def test_the_callables_are_this_interpreters_own(compilers):
    assert os.path.basename(build.CALL_PATH) == "_pycall" + sysconfig.get_config_var("EXT_SUFFIX")
    build.build(force=True)
    assert [cmd[0] for cmd in compilers] == ["nvcc", "g++"] and build.CALL_PATH in compilers[1]


def test_a_compiler_that_fails_is_an_error(monkeypatch):
    def fail(cmd):
        if cmd[0] == "g++":
            raise subprocess.CalledProcessError(1, cmd)

    monkeypatch.setattr(subprocess, "check_call", fail)
    with pytest.raises(subprocess.CalledProcessError):
        build.build(force=True)


def test_calls_without_the_callables(monkeypatch):
    fast = {name: getattr(B._calls(), name) for name in NAMES}
    monkeypatch.setattr(B, "_fast", None)
    monkeypatch.setitem(sys.modules, "paper_2308_14352_b200._pycall", None)   # an import of it fails
    monkeypatch.delattr(sys.modules["paper_2308_14352_b200"], "_pycall", raising=False)
    for name in NAMES:
        good = _arguments(name)
        for i, j in itertools.combinations(range(len(good)), 2):
            a = list(good)
            for k in (i, j):
                a[k] = None if not isinstance(a[k], int) or a[k] > 2 else a[k]
            assert getattr(B._calls(), name)(*a) == fast[name](*a), (name, i, j)
    with pytest.raises(B.EmoeError) as e:
        B.emoe_combine(None, B.emoe_dispatch_desc(64, 4, 2, B.DTYPE_BF16, B.DTYPE_F32, 0, 0, 0), 4096, 4, 4096, None, 4096)
    assert e.value.status == B.ERR_INVALID_ARG
