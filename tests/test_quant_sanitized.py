"""The 8-bit sequence cache's argument checks and plans (seq.cpp) under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): the bad-argument cases of tests/test_quant_checks.py, driven in
a child interpreter against a host-only build, must return the same statuses, and what a decode call
uses of its workspace lies inside the size that it asks for."""
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
import test_quant_checks as t
from paper_2605_30519_amd import omnimem as om

raw = ctypes.CDLL({so!r})
shim = om._configure(raw, required=False)
t.abi = lambda: shim
t.test_cache_arguments()
t.test_decode_arguments()
t.test_append_arguments()
t.test_read_arguments()
t.test_copy_arguments()
print("checks ok")
out = (ctypes.c_int64 * 9)()
taken = refused = lines = 0
big = 2 ** 31 - 1
for heads in (1, 3, 256, 511, 1024, 1 << 17, 1 << 20):
    for G in (1, 5, 16, 17, 32, 33, 100):
        if heads * G > big:
            continue
        for m in (1, 11, 20, 21, 28, 29, 1000, 1 << 15, 1 << 21, (1 << 25) - 100, (1 << 30) - 32):
            for S in (1, 64, 4680):
                for d in (64, 128):
                    for n in (1, 3, 4096):
                        for window in (0, 1, 1560, 5000, big):
                            c = t.cache(num_heads=heads, head_dim=d, num_seqs=n, max_blocks=m, chunk_tokens=S, num_pages=1)
                            size = shim.omnimem_decode_quant_workspace_bytes(ctypes.byref(c), heads * G, window)
                            if raw.shim_decode_quant_plan(ctypes.byref(c), heads * G, window, out) != 0:
                                assert size == 0
                                refused += 1
                                continue
                            taken += 1
                            split, wgs, items, units, shares, at, starts, total, records = out
                            assert size == total and wgs >= 1
                            if window:   # its tokens lie in runs of a chunk, a run of t in t / 64 + 2 blocks at most
                                units = min(units, window // 64 + 2 * (1 if S == 64 else window // S + 2))
                            if split == 0:
                                lines += 1
                                assert -(-items * (units + 3) // wgs) < 2 ** 31, (heads, G, m, S, d, n)
                                assert at % 256 == 0 and at + shares <= starts and starts % 256 == 0 and starts + records <= total
                            else:
                                assert total == 256 and wgs * (4 if split == 2 else 1) >= items
assert taken > 2000 and refused > 500 and lines > 500, (taken, refused, lines)
print("plans ok")
'''


def test_checks_and_plans_under_asan_and_ubsan(tmp_path):
    asan = _runtime("libasan.so")
    if asan is None:
        pytest.skip("gcc's AddressSanitizer runtime is not installed")
    so = tmp_path / "quant_shim.so"
    subprocess.check_call(["g++", "-O1", "-g", "-std=c++17", "-fPIC", "-shared", "-fno-omit-frame-pointer",
                           "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-o", str(so),
                           os.path.join(HERE, "quant_shim.cpp"),
                           os.path.join(ROOT, "paper_2605_30519_amd", "csrc", "seq.cpp")])
    env = dict(os.environ, LD_PRELOAD=asan, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([sys.executable, "-c", CHILD.format(repo=ROOT, tests=HERE, so=str(so))], env=env, capture_output=True,
                       text=True, timeout=600)
    assert r.returncode == 0 and "checks ok" in r.stdout and "plans ok" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])
