"""The binding's two ways of marshalling, for the prompt attention, the 8-bit cache and the pages (no GPU: the calls are refused before
they launch anything)."""
import subprocess
import sys

import pytest

import paper_2605_20022_b200 as fd
from paper_2605_20022_b200 import _build
from test_marshal import Pointer

# (name, arguments in front of the stream): every one is refused by the library itself, which knows no context NULL
CALLS = [("fd_attn_prompt", [None, 1, 1, 1, None, 8, None, None, 8, None, None, None]),
         ("fd_kv_append_fp8", [None, 1, 1, None, None, None, 1, None, None, None]),
         ("fd_kv_read_fp8", [None, 1, 1, None, 1, None, None, None, None, None]),
         ("fd_attn_draft_verify_fp8", [None, 1, 1, None, None, 1, None, None, None, None, None, None]),
         ("fd_kv_fork", [None, 1, None, None, 1] + [None] * 6 + [1, None, None]),
         ("fd_kv_free", [None, 1, None, 1] + [None] * 6 + [1]),
         ("fd_kv_compact", [None, 1, None, None, None, None, 1, None, 1, None, None, None]),
         ("fd_kv_copy_pages", [None, 1, None, None, None, None, 1, fd.FD_KV_BF16])]


@pytest.mark.parametrize("name,args", CALLS)
def test_native_marshalling_and_ctypes_agree(name, args):
    import ctypes
    lib = fd.load()
    seen = []
    kinds = getattr(lib, name).argtypes
    assert len(kinds) == len(args) + 1
    for way in (fd._CtypesMarshal(lib), fd._load_native()):
        assert getattr(way, name)(*args, None) == fd.FD_ERR_INVALID_ARG
        with pytest.raises((TypeError, ValueError)):
            getattr(way, name)(*args)                      # one too few
    record = ctypes.CFUNCTYPE(ctypes.c_int, *kinds)(lambda *a: seen.append(a) or 7)
    record.argtypes = kinds
    values = [Pointer(64 + i) if k is ctypes.c_void_p else i for i, k in enumerate(kinds)]
    assert fd._CtypesMarshal._call(record)(*values) == 7
    assert seen == [tuple(64 + i if k is ctypes.c_void_p else i for i, k in enumerate(kinds))]


def test_every_call_works_without_the_native_marshalling():
    code = f"""
import sys
sys.modules["paper_2605_20022_b200._marshal"] = None    # as on an interpreter that it was not built for
import paper_2605_20022_b200 as fd
for name, args in {CALLS!r}:
    assert getattr(fd, name)(*args, stream=0, raise_on_error=False) == fd.FD_ERR_INVALID_ARG, name
    try:
        getattr(fd, name)(*args, stream=0)
    except RuntimeError as e:
        assert name in str(e)
    else:
        raise AssertionError(name)
assert isinstance(fd._native, fd._CtypesMarshal)
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=_build.ROOT)
