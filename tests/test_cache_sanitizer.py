"""The extension that marshals the calls over a paged cache, built with UBSan, under the tests of what it hands on and refuses."""

import os
import shutil
import subprocess
import sys
import sysconfig

import pytest

from tests.test_host_sanitizers import CSRC, ROOT

PLUGGED = """
import ctypes as C, importlib.util, sys
import pytest
from paper_2407_17678_amd import binding as B
spec = importlib.util.spec_from_file_location("_marshal", sys.argv[1])
calls = importlib.util.module_from_spec(spec)
spec.loader.exec_module(calls)
calls.bind(*(C.cast(getattr(B.lib(), n), C.c_void_p).value for n in B._MARSHALLED))
calls.bind_cache(*(C.cast(getattr(B.lib(), n), C.c_void_p).value for n in B._CACHE_CALLS))
B._calls = calls
code = pytest.main(["-q", "-p", "no:cacheprovider", "tests/test_cache_binding.py", "tests/test_cache_host.py", "-k", "arrives or binding or refused or fit"])
assert B._calls is calls
sys.exit(code)
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_marshalling_of_cache_calls_under_ubsan(tmp_path):
    ext = tmp_path / "_marshal.so"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fPIC", "-shared", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-static-libubsan",
           "-I", sysconfig.get_paths()["include"], os.path.join(CSRC, "marshal.cpp"), "-o", str(ext)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([sys.executable, "-c", PLUGGED, str(ext)], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-2000:])
    assert "passed" in r.stdout
