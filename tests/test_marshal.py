"""The binding with and without its native argument marshalling (no GPU: the calls are refused before they launch anything)."""
import importlib
import os
import subprocess
import sys

import pytest

import paper_2605_20022_b200 as fd
from paper_2605_20022_b200 import _build

# (name, arguments in front of the stream): every one is refused by the library itself, which knows no context NULL
CALLS = [("fd_kv_reserve", [None, 1, 1] + [None] * 10 + [1, None, None]),
         ("fd_qk_norm_rope_append", [None, 1, None, 8, None, None, 1e-6, None, 1, 16, 0, None, None, None, None, 1, fd.FD_KV_BF16, 1.0, 1.0]),
         ("fd_kv_append_fp4", [None, 1, 1, None, None, None, 1, None, None, None, 1.0, 1.0]),
         ("fd_kv_read_fp4", [None, 1, 1, None, 1, None, None, None, 1.0, 1.0, None, None]),
         ("fd_attn_draft_verify_fp4", [None, 1, 1, None, None, 1, None, None, None, None, None, 1.0, 1.0, None])]


class Pointer:
    """What the binding takes for a tensor."""

    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


@pytest.mark.parametrize("name,args", CALLS)
def test_native_marshalling_and_ctypes_agree(name, args):
    import ctypes
    lib = fd.load()
    seen = []
    kinds = getattr(lib, name).argtypes
    as_ctypes = fd._CtypesMarshal(lib)
    for way in (as_ctypes, fd._load_native()):
        assert getattr(way, name)(*args, None) == fd.FD_ERR_INVALID_ARG
        with pytest.raises((TypeError, ValueError)):
            getattr(way, name)(*args)                      # one too few
    record = ctypes.CFUNCTYPE(ctypes.c_int, *kinds)(lambda *a: seen.append(a) or 7)
    record.argtypes = kinds
    values = [Pointer(64 + i) if k is ctypes.c_void_p else float(i) if k is ctypes.c_float else i for i, k in enumerate(kinds)]
    assert fd._CtypesMarshal._call(record)(*values) == 7
    assert seen == [tuple(64 + i if k is ctypes.c_void_p else i for i, k in enumerate(kinds))]


def test_every_call_works_without_the_native_marshalling():
    code = f"""
import sys
sys.modules["paper_2605_20022_b200._marshal"] = None    # as on an interpreter that it was not built for
import paper_2605_20022_b200 as fd
assert fd.status_string(0) == "FD_OK" and fd.fd_plan_ranges_host([300], [4], 2, 3)[-1] == 6
for name, args in {CALLS!r}:
    assert getattr(fd, name)(*args, stream=0, raise_on_error=False) == fd.FD_ERR_INVALID_ARG, name
assert isinstance(fd._native, fd._CtypesMarshal)
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=_build.ROOT)


@pytest.mark.parametrize("error", [FileNotFoundError("gcc"), subprocess.CalledProcessError(1, "gcc")])
def test_library_builds_without_a_c_compiler_or_python_headers(error, tmp_path, monkeypatch):
    _build.build()                                         # (nothing of the library is out of date below)

    def run(cmd, **kw):
        assert cmd[0] == "gcc"
        raise error

    monkeypatch.setattr(_build, "MARSHAL", str(tmp_path / "_marshal.so"))
    monkeypatch.setattr(_build.subprocess, "run", run)
    with pytest.warns(UserWarning, match="ctypes"):
        assert _build.build() == _build.SO and os.path.exists(_build.SO)


def test_the_package_was_built_with_it():
    """Where there is a compiler the native form is the one in use."""
    assert importlib.import_module("paper_2605_20022_b200._marshal") is fd._load_native()
