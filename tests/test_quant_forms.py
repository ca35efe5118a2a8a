"""Which form the 8-bit attention of more than 16 query heads a key head takes, pairs of waves with a column tile each
or both tiles in one wave, against the times of both (CPU only)."""
import ctypes
import os
import subprocess

import pytest

from conftest import ROOT
from paper_2605_30519_amd import omnimem as om

FAKE = 0x10000
BF16, F32 = 0, 1


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("forms") / "quant_form_shim.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(ROOT, "tests", "quant_form_shim.cpp"),
                    os.path.join(ROOT, "paper_2605_30519_amd", "csrc", "seq.cpp"), "-o", so], check=True)
    return ctypes.CDLL(so)


def form(shim, dtype, n, heads, m, window, d, G=24):
    t = om.omnimem_seq_table_t(n, m, 64, 64, 1, FAKE, FAKE)
    c = om.omnimem_seq_cache_quant_t(t, heads, d, FAKE, FAKE, FAKE)
    out = (ctypes.c_int64 * 8)()
    assert shim.shim_decode_form(ctypes.byref(c), dtype, heads * G, window, out) == 0
    return list(out)


# 24 query heads a key head, kernels and join in a graph: type, sequences, key heads, tokens of the longest, window, dims,
# us in pairs, us with both tiles in a wave
WINDOWS = [
    (BF16, 16, 8, 120000, 1560, 128, 27.3, 31.0),
    (BF16, 40, 8, 40000, 5000, 128, 114.4, 92.9),
    (BF16, 24, 8, 60000, 20000, 128, 229.3, 181.9),
    (BF16, 16, 8, 89600, 5350, 128, 62.8, 52.5),
    (BF16, 16, 16, 100000, 4000, 64, 47.5, 43.5),
    (BF16, 16, 8, 44800, 2560, 64, 27.8, 30.2),
    (F32, 16, 8, 120000, 1560, 128, 31.4, 38.7),
    (F32, 16, 16, 100000, 4000, 64, 53.8, 51.6),
    (F32, 16, 8, 44800, 2560, 64, 32.1, 34.7),
    (F32, 24, 8, 60000, 20000, 128, 261.4, 254.2),
]


@pytest.mark.parametrize("dtype,n,heads,hi,window,d,pairs,both", WINDOWS)
def test_windows(shim, dtype, n, heads, hi, window, d, pairs, both):
    """The rule goes by what a window leaves, not by the table: the faster form, where they differ."""
    split, rows, pair, *_ = form(shim, dtype, n, heads, -(-hi // 64) + 1, window, d)
    assert (split, rows) == (0, 32) and bool(pair) == (pairs < both)


# the same without a window: type, sequences, key heads, bytes of capacity / 2^20, dims, us in pairs, us with both in a wave;
# lengths from an eighth of the capacity to all of it, evenly spaced on a logarithmic scale, or (7 sequences) all of it
TABLES = [
    (F32, 16, 8, 256, 128, 46.6, 52.8),
    (F32, 16, 8, 512, 128, 74.3, 79.0),
    (F32, 40, 8, 256, 128, 49.6, 63.0),
    (F32, 40, 8, 768, 128, 100.5, 118.2),
    (F32, 7, 8, 256, 128, 79.8, 82.4),
    (F32, 7, 8, 768, 128, 207.1, 203.5),
    (F32, 16, 8, 512, 64, 74.9, 67.2),
    (F32, 40, 8, 384, 64, 64.6, 61.2),
    (F32, 16, 8, 64, 64, 23.7, 25.6),
    (BF16, 16, 8, 384, 128, 55.0, 50.4),
    (BF16, 16, 8, 192, 128, 33.2, 38.0),
    (BF16, 40, 8, 512, 128, 71.5, 67.0),
    (BF16, 40, 8, 192, 128, 37.1, 43.6),
    (BF16, 16, 8, 384, 64, 51.2, 45.8),
    (BF16, 40, 8, 128, 64, 30.0, 32.0),
]


@pytest.mark.parametrize("dtype,n,heads,mb,d,pairs,both", TABLES)
def test_tables(shim, dtype, n, heads, mb, d, pairs, both):
    split, rows, pair, *_ = form(shim, dtype, n, heads, mb * 2 ** 20 // (2 * n * heads * 64 * d) + 1, 0, d)
    assert (split, rows) == (0, 32) and bool(pair) == (pairs < both)


def test_the_workspace_serves_both_types(shim):
    """Its size is asked for without a type, so every type's regions lie inside it."""
    forms = set()
    for heads in (1, 8, 9, 40, 300):
        for n in (1, 16, 40):
            for m in (30, 200, 400, 800, 3000, 20000):
                for window in (0, 1560, 40000):
                    for d in (64, 128):
                        for G in (1, 17, 40):
                            sizes = set()
                            for dtype in (BF16, F32):
                                split, _, pair, wgs, at, shares, starts, need = form(shim, dtype, n, heads, m, window, d, G)
                                if split == 0:
                                    assert at + shares <= starts and starts + 24 * wgs <= need   # a record has 24 bytes
                                    forms.add((dtype, pair))
                                sizes.add(need)
                            assert len(sizes) == 1
    assert len(forms) == 4


def test_a_window_that_bounds_nothing_is_none(shim):
    for dtype in (BF16, F32):
        for d in (64, 128):
            for m in (40, 300, 1000, 5000):
                want = form(shim, dtype, 8, 8, m, 0, d)
                assert form(shim, dtype, 8, 8, m, 64 * m, d) == want == form(shim, dtype, 8, 8, m, 2 ** 31 - 1, d)
