"""The 8-bit sequence cache's refusals, on the CPU: the C ABI's statuses for bad arguments (nothing is
launched), its workspace sizes, and the binding's checks of tensors, each with a message that names
the argument.  CPU tensors of the right shape are refused last."""
import ctypes

import pytest
import torch

from paper_2605_30519_amd import omnimem as om
from test_seq_checks import BIG, EINVAL, EUNSUP, EWS, FAKE, OK, TABLE_CASES, refused, table

BF, F32C = 0, 1


def abi():
    """The library the C cases run against; the sanitizer test swaps in a host-only build."""
    return om.lib()


def cache(num_heads=2, head_dim=64, k_pages=FAKE, v_pages=FAKE, scales=FAKE, **kw):
    return om.omnimem_seq_cache_quant_t(table(**kw), num_heads, head_dim, k_pages, v_pages, scales)


CACHE_CASES = [
    (dict(head_dim=96), EUNSUP), (dict(num_heads=0), EINVAL), (dict(num_heads=2 ** 20 + 1), EINVAL), (dict(k_pages=0), EINVAL),
    (dict(v_pages=0), EINVAL), (dict(k_pages=FAKE + 8), EINVAL), (dict(v_pages=FAKE + 4), EINVAL), (dict(scales=0), EINVAL),
    (dict(scales=FAKE + 4), EINVAL), (dict(num_pages=BIG, num_heads=2 ** 20, head_dim=128), EINVAL),   # past 2^40 elements
]


def test_cache_arguments():
    L = abi()
    for kw, want in TABLE_CASES + CACHE_CASES:
        c = ctypes.byref(cache(**kw))
        assert L.omnimem_decode_attn_quant(c, BF, FAKE, 128, 2, 0, 0.1, FAKE, None, FAKE, 1 << 30, None) == want, kw
        assert L.omnimem_append_kv_quant(c, BF, FAKE, 128, FAKE, 128, 3, None, None) == want, kw
        assert L.omnimem_read_kv_quant(c, BF, 3, None, None, FAKE, FAKE, None) == want, kw
    c = ctypes.byref(cache())
    for dtype in (-1, 2, 3):
        assert L.omnimem_decode_attn_quant(c, dtype, FAKE, 128, 2, 0, 0.1, FAKE, None, FAKE, 1 << 30, None) == EUNSUP
        assert L.omnimem_append_kv_quant(c, dtype, FAKE, 128, FAKE, 128, 3, None, None) == EUNSUP
        assert L.omnimem_read_kv_quant(c, dtype, 3, None, None, FAKE, FAKE, None) == EUNSUP
    assert L.omnimem_decode_attn_quant(None, BF, FAKE, 128, 2, 0, 0.1, FAKE, None, FAKE, 1 << 30, None) == EINVAL
    assert L.omnimem_append_kv_quant(None, BF, FAKE, 128, FAKE, 128, 3, None, None) == EINVAL
    assert L.omnimem_read_kv_quant(None, BF, 3, None, None, FAKE, FAKE, None) == EINVAL


def test_decode_arguments():
    L = abi()
    c = cache(max_blocks=1000)
    need = L.omnimem_decode_quant_workspace_bytes(ctypes.byref(c), 4, 0)
    assert need > 256 and need % 256 == 0

    def call(dtype=BF, q=FAKE, stride=256, heads=4, window=0, scale=0.1, out=FAKE, lse=FAKE, ws=FAKE, n=need, c=c):
        return L.omnimem_decode_attn_quant(ctypes.byref(c), dtype, q, stride, heads, window, scale, out, lse, ws, n, None)

    for kw in (dict(q=0), dict(q=FAKE + 8), dict(out=0), dict(out=FAKE + 4), dict(lse=FAKE + 2), dict(heads=3),
               dict(heads=0), dict(heads=-2), dict(stride=255), dict(stride=260), dict(dtype=F32C, stride=258),
               dict(stride=-256), dict(stride=2 ** 41), dict(window=-1), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(ws=0), dict(ws=FAKE + 16)):
        assert call(**kw) == EINVAL, kw
    assert call(n=need - 1) == EWS
    assert L.omnimem_decode_attn_quant(ctypes.byref(cache(num_seqs=0, page_table=0, seq_lens=0)), BF, None, 256, 4, 0, 0.1, None,
                                       None, None, 0, None) == OK
    bare = cache(max_blocks=1000, page_table=0, seq_lens=0, k_pages=0, v_pages=0, scales=0)
    size = L.omnimem_decode_quant_workspace_bytes
    assert size(ctypes.byref(bare), 4, 0) == need
    assert size(ctypes.byref(bare), 3, 0) == 0 == size(None, 4, 0) == size(ctypes.byref(bare), 4, -1)
    assert 256 < size(ctypes.byref(bare), 4, 40000) <= need
    assert size(ctypes.byref(bare), 4, 1) == 256 == size(ctypes.byref(cache()), 4, 0)
    assert size(ctypes.byref(cache(num_seqs=BIG, max_blocks=2 ** 20)), 4, 0) == 0


def test_append_arguments():
    L = abi()

    def call(dtype=BF, k=FAKE, ks=128, v=FAKE, vs=128, tokens=3, starts=FAKE, c=cache()):
        return L.omnimem_append_kv_quant(ctypes.byref(c), dtype, k, ks, v, vs, tokens, starts, None)

    for kw in (dict(k=0), dict(v=0), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(ks=127), dict(vs=132),
               dict(dtype=F32C, ks=130), dict(ks=-128), dict(tokens=-1), dict(starts=FAKE + 1), dict(starts=None, tokens=2),
               dict(vs=2 ** 41)):
        assert call(**kw) == EINVAL, kw
    assert call(tokens=0, k=0, v=0) == OK
    assert call(c=cache(num_seqs=0, page_table=0, seq_lens=0)) == OK


def test_read_arguments():
    L = abi()

    def call(tokens=3, starts=FAKE, first=FAKE, k=FAKE, v=FAKE, c=cache()):
        return L.omnimem_read_kv_quant(ctypes.byref(c), BF, tokens, starts, first, k, v, None)

    for kw in (dict(tokens=-1), dict(tokens=2, starts=None), dict(starts=FAKE + 2), dict(first=FAKE + 1), dict(k=0), dict(v=0),
               dict(k=FAKE + 8), dict(v=FAKE + 4)):
        assert call(**kw) == EINVAL, kw
    assert call(tokens=0, k=0, v=0) == OK
    assert call(c=cache(num_seqs=0, page_table=0, seq_lens=0), starts=None, tokens=0) == OK


def test_copy_arguments():
    L = abi()

    def call(k=FAKE, v=FAKE, s=FAKE, pages=10, heads=2, B=64, d=64, layers=2, step=81920, sstep=160, pairs=FAKE, count=FAKE,
             most=4):
        return L.omnimem_copy_pages_quant(k, v, s, pages, heads, B, d, layers, step, sstep, pairs, count, most, None)

    for kw in (dict(k=0), dict(v=0), dict(s=0), dict(k=FAKE + 8), dict(v=FAKE + 8), dict(s=FAKE + 4), dict(pages=-1),
               dict(pages=2 ** 31), dict(heads=0), dict(heads=2 ** 21), dict(layers=-1), dict(step=81904), dict(step=81921),
               dict(step=-16), dict(sstep=152), dict(sstep=161), dict(sstep=-8), dict(sstep=2 ** 45), dict(pairs=0),
               dict(pairs=FAKE + 2), dict(count=FAKE + 1), dict(most=-1), dict(pages=BIG, heads=2 ** 20, B=128, d=128)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(B=32), dict(d=32), dict(B=0)):
        assert call(**kw) == EUNSUP, kw
    for kw in (dict(pages=0, k=0, v=0, s=0), dict(layers=0), dict(most=0, pairs=0)):
        assert call(**kw) == OK, kw


# ------------------------------------------------------------------------- the binding

H, D, B, N, M, P = 2, 64, 64, 3, 4, 12
I32, BF16, F32, F8 = torch.int32, torch.bfloat16, torch.float32, torch.float8_e4m3fn


def quant_cache():
    pages = torch.zeros((P, H, B, D), dtype=torch.uint8)
    return om.SeqKVCacheQuant(pages.view(F8), pages.clone().view(F8), torch.ones((P, H, 2)), torch.zeros((N, M), dtype=I32),
                              torch.zeros(N, dtype=I32))


def rows(n=N, h=H, d=D, dtype=BF16):
    return torch.zeros((n, h, d), dtype=dtype)


def test_binding_cache():
    def bad(match, error=ValueError, **kw):
        c = quant_cache()
        for name, t in kw.items():
            setattr(c, name, t)
        refused(match, c.descriptor, error=error)
        refused(match, c.packed, error=error)
        refused(match, om.omnimem_decode_attn_quant, c, rows(), error=error)
        refused(match, om.omnimem_append_kv_quant, c, rows(), rows(), error=error)
        refused(match, om.omnimem_read_kv_quant, c, N, error=error)

    c = quant_cache()
    bad("must be torch.float8_e4m3fn", TypeError, k_pages=c.k_pages.view(torch.uint8))
    bad("must be torch.float8_e4m3fn", TypeError, v_pages=c.v_pages.view(torch.uint8).view(torch.float8_e5m2))
    bad("share one", v_pages=c.v_pages[:-1])
    bad("share one", k_pages=c.k_pages[0], v_pages=c.v_pages[0])
    bad("cache tensors must be contiguous", k_pages=torch.zeros((H, P, B, D), dtype=torch.uint8).view(F8).transpose(0, 1))
    bad("scales must have shape", scales=torch.ones((P, H)))
    bad("scales must be torch.float32", scales=torch.ones((P, H, 2), dtype=torch.float64))
    bad("scales must be contiguous", scales=torch.ones((P, 2, H)).transpose(1, 2))
    bad("page_table must be torch.int32", page_table=c.page_table.long())
    bad("page_table must be contiguous", page_table=torch.zeros((M, N), dtype=I32).t())
    bad(r"page_table must be an \[N, max_blocks\] tensor", page_table=torch.zeros((N, M, 1), dtype=I32))
    bad("seq_lens must have shape", seq_lens=torch.zeros(N + 1, dtype=I32))
    bad("out of range", chunk_tokens=2 ** 32 + 64)
    bad("the cache must live on a GPU")


def test_binding_calls():
    """Shapes and types are looked at behind the cache, whose CPU tensors end every call here: these
    checks are called by themselves."""
    like = quant_cache().k_pages
    for f in (om._quant_rows, om._rows_stride):
        args = (lambda t, *a: f(t, *a)) if f is om._quant_rows else (lambda t, *a: f("q", t, *a))
        assert args(rows(), H, like, BF16) == H * D
        assert args(torch.zeros((N, 3, H, D))[:, 1], H, like, F32) == 3 * H * D
    for t, heads, dtype in ((rows()[0], None, BF16), (rows(d=32), None, BF16), (rows(), H, F32), (rows(h=3), H, BF16),
                            (torch.zeros((N, D, H), dtype=BF16).transpose(1, 2), None, BF16)):
        assert om._quant_rows(t, heads, like, dtype) == 0
        refused("q must", om._rows_stride, "q", t, heads, like, dtype)
    assert om._quant_rows(rows(n=1), H, like, BF16) == 0 and om._rows_stride("q", rows(n=1), H, like, BF16) == H * D
    refused("k must be a bf16 or fp32 tensor", om.omnimem_append_kv_quant, quant_cache(), rows(dtype=torch.float16), rows())
    refused("q must be a bf16 or fp32 tensor", om.omnimem_decode_attn_quant, quant_cache(), None)
    refused("k and v must have one row", om._check_starts, None, N + 1, N, "k and v")
    refused("starts must have shape", om._check_starts, torch.zeros(N, dtype=I32), N, N, "k and v")
    refused("starts must be torch.int32", om._check_starts, torch.zeros(N + 1), N, N, "k and v")


def test_binding_copy():
    c = quant_cache()
    f, k, v, s = om.omnimem_copy_pages_quant, c.k_pages, c.v_pages, c.scales
    pairs = torch.zeros((2, 2), dtype=I32)
    refused("k_pages must be", f, k[0], v[0], s[0], pairs)
    refused("k_pages must be torch.float8_e4m3fn", f, k.float(), v, s, pairs)
    refused("v_pages must be torch.float8_e4m3fn", f, k, None, s, pairs)
    refused("v_pages must have shape", f, k, v[:-1], s, pairs)
    refused("scales must have shape", f, k, v, s[:, :1], pairs)
    refused("scales must be torch.float32", f, k, v, s.double(), pairs)
    refused("k_pages must be contiguous", f, k[:, :1], v[:, :1], s[:, :1], pairs)
    six = (2, 6, H, B, D)
    refused("distance between layers", f, k.view(six), torch.zeros((2, 2, 6, H, B, D), dtype=torch.uint8).view(F8)[:, 0],
            s.view(2, 6, H, 2), pairs)
    refused(r"pairs must be an \[n, 2\] tensor", f, k, v, s, pairs[0])
    refused("pairs must have shape", f, k, v, s, torch.zeros((2, 3), dtype=I32))
    refused("pairs must be torch.int32", f, k, v, s, pairs.long())
    refused("count must be an int32 tensor", f, k, v, s, pairs, torch.zeros(1, dtype=torch.int64))
    refused("k_pages must live on a GPU", f, k, v, s, pairs)


def test_the_packed_descriptor_is_the_structure():
    """packed's fields lie where the structure's do."""
    fields = (3, 4, 64, 100, 12, 0x1000, 0x2000, 2, 128, 0x3000, 0x4000, 0x5000)
    t = om.omnimem_seq_table_t(*fields[:7])
    assert om._pack_quant(*fields) == bytes(om.omnimem_seq_cache_quant_t(t, *fields[7:]))
