"""The sequence cache's work plans on the CPU, from a host-only build: what a call uses of its
workspace lies inside the size that it asks for."""
import ctypes
import os
import subprocess
import sys

import pytest

from conftest import ROOT
from paper_2605_30519_amd import omnimem as om

FAKE = 0x10000  # aligned, never dereferenced


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plans") / "seq_plan_shim.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(ROOT, "tests", "seq_plan_shim.cpp"),
                    os.path.join(ROOT, "paper_2605_30519_amd", "csrc", "seq.cpp"), "-o", so], check=True)
    return ctypes.CDLL(so)


def table(n, m, pages):
    return om.omnimem_seq_table_t(n, m, 64, 64, pages, FAKE, FAKE)


@pytest.mark.parametrize("new", [0, 1, 5, 1300])
@pytest.mark.parametrize("n,m,pages", [(3, 10, 30), (256, 65, 4000), (2000, 2, 100), (3, 10, 16385), (7, 70, 1 << 20),
                                       (0, 5, 20000), (5000, 9, 0)])
def test_update_stays_inside_its_workspace(shim, n, m, pages, new):
    """The bitmaps, a word per page and the rows' records lie one behind the other; without new rows
    only the first bitmap has a place, and nothing else may be used."""
    out = (ctypes.c_int64 * 9)()
    assert shim.shim_update_plan(ctypes.byref(table(n, m, pages)), new, out) == 0
    one, growing, words, held, tail, first, rows, total, record = out
    rows_here = new or n
    assert one == (pages <= 16384 and rows_here <= 1024 and rows_here * m <= 8192)
    assert growing == (new > 0) and words == -(-pages // 32)
    if one:
        return                                                   # all in one workgroup's LDS
    ends = [(held, 4 * words)]
    if growing:
        ends += [(tail, 4 * words), (first, 4 * pages), (rows, record * new)]
    for (at, size), behind in zip(ends, [a for a, _ in ends[1:]] + [total]):
        assert at % 256 == 0 and at + size <= behind


LARGE_WINDOWS = r'''
import ctypes, sys
sys.path[:0] = [{repo!r}]
from paper_2605_30519_amd import omnimem as om

f = om._configure(ctypes.CDLL({so!r}), required=False).omnimem_decode_workspace_bytes
big = 2 ** 31 - 1
for n, m in ((2, 5000), (4, 100000), (700, 3)):
    for dtype, d in ((0, 64), (0, 128), (1, 64), (1, 128)):
        for B in (64, 128):
            for S in (1, 2, 3, 63, 64, 65, 100, 4680, big):
                cache = om.omnimem_seq_cache_t(om.omnimem_seq_table_t(n, m, B, S, 30, None, None), dtype, 2, d, None, None)
                whole = f(ctypes.byref(cache), 4, 0)
                for window in (big, big - 1, big - 2, big - 3, 2 ** 30):
                    assert f(ctypes.byref(cache), 4, window) == whole, (n, m, dtype, d, B, S, window)
print("windows ok")
'''


def test_a_window_past_every_row_is_no_window(tmp_path):
    """The largest windows with chunks of a token and more take what the whole rows take, with no
    signed overflow on the way (UndefinedBehaviorSanitizer, in a child interpreter)."""
    so = str(tmp_path / "seq_shim.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-fsanitize=undefined", "-static-libubsan",
                    "-fno-sanitize-recover=undefined", os.path.join(ROOT, "tests", "seq_shim.cpp"),
                    os.path.join(ROOT, "paper_2605_30519_amd", "csrc", "seq.cpp"), "-o", so], check=True)
    r = subprocess.run([sys.executable, "-c", LARGE_WINDOWS.format(repo=ROOT, so=so)], capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0 and "windows ok" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])


def test_a_share_of_the_line_is_counted_in_31_bits(shim):
    """Whatever the checks accept leaves every workgroup of a decode call a share below 2^31 units: an
    item counts its units and three more."""
    out = (ctypes.c_int64 * 4)()
    taken = refused = 0
    for heads in (1, 256, 257, 511, 512, 513, 1024, 4096, 1 << 17, 1 << 18, 1 << 19, 1 << 20):
        for m in (1, 11, 1000, 1 << 15, 1 << 20, 1 << 21, 1 << 22, (1 << 25) - 100, 1 << 29, (1 << 30) - 32):
            for S in (1, 64):
                for dtype, d in ((0, 64), (1, 64)):
                    for n in (1, 3):
                        cache = om.omnimem_seq_cache_t(om.omnimem_seq_table_t(n, m, 64, S, 1, FAKE, FAKE), dtype, heads, d,
                                                       FAKE, FAKE)
                        if shim.shim_decode_plan(ctypes.byref(cache), heads, 0, out) != 0:
                            refused += 1
                            continue
                        taken += 1
                        split, wgs, items, units = out
                        assert split != 0 or -(-items * (units + 3) // wgs) < 2 ** 31, (heads, m, S, dtype, n)
    assert taken > 200 and refused > 50
