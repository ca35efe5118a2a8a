"""The sequence cache's argument checks (seq.cpp) under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): the bad-argument cases of tests/test_seq_checks.py,
driven in a child interpreter against a host-only build, must return the same statuses."""
import os
import subprocess
import sys

import pytest

from conftest import ROOT
from test_host_sanitized import _runtime

HERE = os.path.dirname(os.path.abspath(__file__))
CHILD = r'''
import ctypes, sys
sys.path[:0] = [{repo!r}, {tests!r}]
import test_seq_checks as t
from paper_2605_30519_amd import omnimem as om

shim = om._configure(ctypes.CDLL({so!r}), required=False)
t.abi = lambda: shim
t.test_cache_arguments()
t.test_decode_arguments()
t.test_append_arguments()
t.test_copy_arguments()
t.test_update_and_compact_arguments()
print("checks ok")
'''


def test_checks_under_asan_and_ubsan(tmp_path):
    asan = _runtime("libasan.so")
    if asan is None:
        pytest.skip("gcc's AddressSanitizer runtime is not installed")
    so = tmp_path / "seq_shim.so"
    subprocess.check_call(["g++", "-O1", "-g", "-std=c++17", "-fPIC", "-shared", "-fno-omit-frame-pointer",
                           "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-o", str(so),
                           os.path.join(HERE, "seq_shim.cpp"),
                           os.path.join(ROOT, "paper_2605_30519_amd", "csrc", "seq.cpp")])
    env = dict(os.environ, LD_PRELOAD=asan, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    code = CHILD.format(repo=ROOT, tests=HERE, so=str(so))
    r = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "checks ok" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])
