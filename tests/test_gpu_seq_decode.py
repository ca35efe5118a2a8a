"""omnimem_decode_attn against fp64: every type, head size, block and chunk size, groups of 1 to
40 query heads, lengths around each border, windows, pages that are not resident, shared pages.
Slots that hold no token of a sequence are NaN in every case."""
import math

import pytest
import torch

import seq_oracle
from parity import say
from paper_2605_30519_amd import (OmniMemError, SeqKVCache, omnimem_decode_attn, omnimem_decode_workspace_bytes,
                                  omnimem_dense_attn)
from paper_2605_30519_amd.omnimem import workspace_tensor

pytestmark = pytest.mark.gpu
NAN = float("nan")
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


def build(dev, dtype, H, d, B, S, lens, seed, extra_blocks=1, spare=3, std=1.0):
    """A cache of the given lengths over shuffled pages, NaN wherever no token lies."""
    g = torch.Generator().manual_seed(seed)
    nb = [seq_oracle.blocks(t, S, B) for t in lens]
    M = max(nb + [0]) + extra_blocks
    P = sum(nb) + spare
    ids = torch.randperm(P, generator=g).tolist()
    table = [[ids.pop() for _ in range(n)] + [-5] * (M - n) for n in nb]
    k = torch.full((P, H, B, d), NAN, dtype=dtype)
    v = torch.full((P, H, B, d), NAN, dtype=dtype)
    for row, t in zip(table, lens):
        if t == 0:
            continue
        block, slot = (torch.tensor(x) for x in zip(*(seq_oracle.place(x, S, B) for x in range(t))))
        page = torch.tensor(row)[block]
        k[page, :, slot] = (std * torch.randn((t, H, d), generator=g)).to(dtype)
        v[page, :, slot] = torch.randn((t, H, d), generator=g).to(dtype)
    cache = SeqKVCache(k.to(dev), v.to(dev), torch.tensor(table, dtype=torch.int32, device=dev).view(len(lens), M),
                       torch.tensor(lens, dtype=torch.int32, device=dev), S)
    return cache, g


def queries(dev, dtype, N, Hq, d, g, std=1.5):
    return (std * torch.randn((N, Hq, d), generator=g)).to(dtype).to(dev)


def check(cache, q, window=0, scale=None, **kw):
    B, d = cache.k_pages.shape[2:]
    out, lse = omnimem_decode_attn(cache, q, scale, window=window, **kw)
    torch.cuda.synchronize()
    O, L, ob, lb = seq_oracle.decode(q, cache.k_pages, cache.v_pages, cache.page_table, cache.seq_lens, B,
                                     cache.chunk_tokens or B, window, scale or 1 / math.sqrt(d))
    got, gl = out.double().cpu(), lse.double().cpu()
    assert not torch.isnan(got).any() and not torch.isnan(gl).any()
    empty = torch.isinf(L)
    assert torch.equal(torch.isinf(gl), empty) and (gl[empty] < 0).all()
    assert (got.transpose(0, 1)[empty] == 0).all()
    over = ((got - O).abs() - ob).max().item()
    assert over <= 0, f"O is {over:.3g} past its bound"
    diff = ((gl - L).abs() - lb)[~empty]
    assert diff.numel() == 0 or diff.max().item() <= 0, f"lse is {diff.max().item():.3g} past its bound"
    return out, lse


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 0]


@pytest.mark.parametrize("dtype,d,B", [(BF16, 128, 64), (BF16, 64, 64), (F32, 128, 64), (F32, 64, 64), (BF16, 128, 128),
                                       (F32, 64, 128)])
@pytest.mark.parametrize("H,G", [(3, 1), (2, 5)])
def test_lengths_around_every_border(dev, dtype, d, B, H, G):
    say(f"decode edges {dtype} d={d} B={B} H={H} G={G}")
    cache, g = build(dev, dtype, H, d, B, B, EDGES, 1)
    check(cache, queries(dev, dtype, len(EDGES), H * G, d, g))


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 128), (BF16, 64), (F32, 64)])
@pytest.mark.parametrize("G", [2, 8, 15, 16, 17, 24, 31, 32, 33, 40])
def test_query_heads_per_key_head(dev, dtype, d, G):
    say(f"decode groups {dtype} d={d} G={G}")
    cache, g = build(dev, dtype, 2, d, 64, 64, [200, 0, 70, 1000], 2)
    check(cache, queries(dev, dtype, 4, 2 * G, d, g))


@pytest.mark.parametrize("dtype,d,B,S", [(BF16, 128, 64, 100), (F32, 64, 64, 130), (BF16, 64, 128, 200), (F32, 128, 128, 70),
                                         (BF16, 128, 64, 1), (BF16, 128, 64, 256), (BF16, 128, 128, 4680)])
def test_chunks_with_partial_blocks(dev, dtype, d, B, S):
    lens = [0, 1, S, S + 1, max(S - 1, 0), 2 * S, 3 * S + 70 % S] if S < 4680 else [4680, 4681, 9000]
    say(f"decode chunks {dtype} d={d} B={B} S={S} lens={lens}")
    cache, g = build(dev, dtype, 2, d, B, S, lens, 3)
    for window in (0, 1, 90):
        check(cache, queries(dev, dtype, len(lens), 4, d, g), window)


@pytest.mark.parametrize("dtype,B,S", [(BF16, 64, 64), (F32, 128, 128), (BF16, 128, 300), (BF16, 64, 4000)])
@pytest.mark.parametrize("window", [1, 16, 63, 64, 65, 200, 1000, 2 ** 31 - 1])
def test_windows(dev, dtype, B, S, window):
    """The tokens before a window, in its first block too, are NaN here."""
    lens = [0, 1, 64, 65, 128, 500, 1100]
    say(f"decode window {dtype} B={B} S={S} window={window}")
    cache, g = build(dev, dtype, 2, 128, B, S, lens, 4)
    rows = cache.page_table.tolist()
    for row, t in zip(rows, lens):
        for x in range(max(0, t - window)):
            b, s = seq_oracle.place(x, S, B)
            cache.k_pages[row[b], :, s] = NAN
            cache.v_pages[row[b], :, s] = NAN
    check(cache, queries(dev, dtype, len(lens), 6, 128, g), window)


def test_pages_not_resident(dev):
    cache, g = build(dev, BF16, 2, 128, 64, 64, [640, 64, 130, 500], 5)
    t = cache.page_table
    t[0, 1] = -1
    t[0, 4] = 2 ** 30           # no such page
    t[0, 9] = cache.k_pages.shape[0]
    t[1, 0] = -1                # nothing left
    t[3, 0:8] = torch.tensor([-1, -1, 3, -1, -1, -1, -1, -1])
    cache.k_pages.nan_to_num_(0.5)
    cache.v_pages.nan_to_num_(0.25)
    out, lse = check(cache, queries(dev, BF16, 4, 4, 128, g))
    assert (out[1] == 0).all() and torch.isinf(lse[:, 1]).all()


def test_lengths_past_the_row_and_below_zero(dev):
    cache, g = build(dev, F32, 1, 64, 64, 64, [128, 100, 64], 6, extra_blocks=0)
    cache.k_pages.nan_to_num_(0.0)
    cache.v_pages.nan_to_num_(1.0)
    cache.seq_lens.copy_(torch.tensor([2 ** 31 - 1, -3, 64]))
    check(cache, queries(dev, F32, 3, 1, 64, g))


def test_sequences_that_share_pages(dev):
    cache, g = build(dev, BF16, 4, 128, 64, 64, [700, 650, 10], 7)
    cache.page_table[1, :10] = cache.page_table[0, :10]
    cache.page_table[2, 0] = cache.page_table[0, 3]
    check(cache, queries(dev, BF16, 3, 8, 128, g))


def test_scores_far_from_zero(dev):
    """Large scores of either sign, and a key whose score is above all others by hundreds."""
    cache, g = build(dev, BF16, 2, 128, 64, 64, [1000, 333], 8, std=6.0)
    q = queries(dev, BF16, 2, 4, 128, g, std=6.0)
    check(cache, q)
    cache, g = build(dev, F32, 2, 64, 64, 64, [1000, 333], 9, std=8.0)
    check(cache, queries(dev, F32, 2, 4, 64, g, std=8.0))


@pytest.mark.parametrize("N,H,G,t", [(1, 1, 1, 100000), (1, 8, 4, 20000), (3, 12, 1, 9000)])
def test_long_sequences_split_over_workgroups(dev, N, H, G, t):
    say(f"decode long N={N} H={H} G={G} t={t}")
    cache, g = build(dev, BF16, H, 128, 64, 64, [t - 17 * i for i in range(N)], 10)
    check(cache, queries(dev, BF16, N, H * G, 128, g))


def test_many_sequences(dev):
    """More sequences than threads in a workgroup, most of them short or empty."""
    lens = [(i * 37) % 90 if i % 3 else 0 for i in range(700)]
    cache, g = build(dev, F32, 1, 64, 64, 64, lens, 11)
    check(cache, queries(dev, F32, 700, 2, 64, g))


@pytest.mark.parametrize("dtype,d,H,G,window", [(BF16, 128, 4, 3, 0), (F32, 64, 8, 20, 0), (BF16, 64, 3, 1, 5), (F32, 128, 4, 17, 90)])
def test_many_short_items(dev, dtype, d, H, G, window):
    """Over a thousand (sequence, head) items of up to two blocks, or of a short window; the last
    workgroup is not full."""
    N = 345 if H == 3 else 260 if H == 4 else 131
    lens = [(i * 29) % 129 for i in range(N)]
    if window:
        lens[7], lens[100] = 400, 129
    say(f"decode short {dtype} d={d} H={H} G={G} window={window}")
    cache, g = build(dev, dtype, H, d, 64, 64, lens, 18, extra_blocks=0)
    check(cache, queries(dev, dtype, N, H * G, d, g), window)


def test_thousands_of_sequences_most_of_them_empty(dev):
    """More sequences than one look at them by a workgroup's lanes, some long, so that shares are joined."""
    lens = [900 if i % 5000 == 17 else 40 if i % 700 == 3 else 0 for i in range(20000)]
    cache, g = build(dev, F32, 1, 64, 64, 64, lens, 19)
    q = queries(dev, F32, len(lens), 1, 64, g)
    out, lse = omnimem_decode_attn(cache, q)
    some = [i for i, t in enumerate(lens) if t] + [0, 1, 19999]
    O, L, ob, lb = seq_oracle.decode(q[some], cache.k_pages, cache.v_pages, cache.page_table[some], cache.seq_lens[some], 64,
                                     64, 0, 0.125)
    assert ((out[some].double().cpu() - O).abs() <= ob).all()
    full = torch.tensor(lens) > 0
    assert (out.cpu()[~full] == 0).all() and (lse.cpu()[:, ~full] == -math.inf).all() and torch.isfinite(lse.cpu()[:, full]).all()


@pytest.mark.parametrize("dtype,d,G,t", [(BF16, 128, 4, 3300), (BF16, 64, 1, 6500), (F32, 128, 3, 3300), (F32, 64, 16, 3300),
                                         (BF16, 128, 20, 3300)])
def test_long_sequences_that_share_most_pages(dev, dtype, d, G, t):
    """Rows that one prompt's pages serve, beside one with its own and two prompts in turn: each
    workgroup's share is long and its pages are shared, or not.  The same pages held once for each
    row give the same bits."""
    say(f"decode shared {dtype} d={d} G={G}")
    base, g = build(dev, dtype, 4, d, 64, 64, [t, t - 900, t - 70], 20)
    src = [0] * 29 + [1] + [2] * 20 + [0, 2] * 7
    table = base.page_table[src].contiguous()
    lens = base.seq_lens[src] - torch.arange(64, dtype=torch.int32, device=dev)
    cache = SeqKVCache(base.k_pages, base.v_pages, table, lens, 64)
    q = queries(dev, dtype, 64, 4 * G, d, g)
    out, lse = omnimem_decode_attn(cache, q)
    own = table.long().clamp(min=0).flatten()
    apart = SeqKVCache(base.k_pages[own], base.v_pages[own],
                       torch.arange(own.numel(), dtype=torch.int32, device=dev).view_as(table), lens, 64)
    out2, lse2 = omnimem_decode_attn(apart, q)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    some = [0, 28, 29, 49, 50, 63]
    O, L, ob, lb = seq_oracle.decode(q[some], cache.k_pages, cache.v_pages, table[some], lens[some], 64, 64, 0, d ** -0.5)
    assert ((out[some].double().cpu() - O).abs() <= ob).all()
    assert ((lse[:, some].double().cpu() - L).abs() <= lb).all()


def test_strided_queries_and_given_buffers(dev):
    cache, g = build(dev, BF16, 2, 128, 64, 64, [100, 300, 5], 12)
    qkv = queries(dev, BF16, 3, 4 * 3, 128, g).view(3, 3, 4, 128)
    q = qkv[:, 1]
    want, wl = check(cache, q)
    out = torch.full((3, 4, 128), NAN, dtype=BF16, device=dev)
    lse = torch.full((4, 3), NAN, device=dev)
    ws = workspace_tensor(omnimem_decode_workspace_bytes(cache, 4), dev)
    ws.fill_(255)
    got, gl = omnimem_decode_attn(cache, q, out=out, lse=lse, workspace=ws)
    assert got is out and torch.equal(out, want) and torch.equal(lse, wl)
    got, none = omnimem_decode_attn(cache, q.contiguous(), want_lse=False)
    assert none is None and torch.equal(got, want)


def test_the_same_call_gives_the_same_bits(dev):
    cache, g = build(dev, BF16, 4, 128, 64, 64, [5000, 20, 900, 0, 77], 13)
    q = queries(dev, BF16, 5, 12, 128, g)
    first = omnimem_decode_attn(cache, q)
    for _ in range(3):
        again = omnimem_decode_attn(cache, q)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


def test_no_sequences(dev):
    cache, _ = build(dev, BF16, 2, 64, 64, 64, [], 14)
    out, lse = omnimem_decode_attn(cache, torch.empty((0, 2, 64), dtype=BF16, device=dev))
    assert out.shape == (0, 2, 64) and lse.shape == (2, 0)


def test_an_empty_pool(dev):
    cache = SeqKVCache(torch.empty((0, 2, 64, 64), device=dev), torch.empty((0, 2, 64, 64), device=dev),
                       torch.zeros((2, 3), dtype=torch.int32, device=dev),
                       torch.tensor([100, 0], dtype=torch.int32, device=dev))
    out, lse = omnimem_decode_attn(cache, torch.ones((2, 2, 64), device=dev))
    assert (out == 0).all() and torch.isinf(lse).all()


def test_another_stream(dev):
    cache, g = build(dev, BF16, 2, 128, 64, 64, [2000, 100], 15)
    q = queries(dev, BF16, 2, 2, 128, g)
    want, wl = omnimem_decode_attn(cache, q)
    torch.cuda.synchronize()
    for stream in (torch.cuda.Stream(device=dev), 0):
        got, gl = omnimem_decode_attn(cache, q, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(gl, wl)


def test_agrees_with_dense_attention_of_one_row(dev):
    """A sequence of whole chunks, as omnimem_dense_attn sees it through SeqKVCache.chunks."""
    cache, g = build(dev, F32, 3, 128, 64, 100, [500], 16)
    cache.k_pages.nan_to_num_(0.0)
    q = queries(dev, F32, 1, 3, 128, g)
    out, lse = check(cache, q)
    dense, dl = omnimem_dense_attn(cache.chunks(0, 5), q, 0, 5)
    # two fp32 sums of 500 terms each, of values of unit size
    assert (out - dense).abs().max() < 2 * 600 * 2 ** -24 * 4 and (lse - dl).abs().max() < 1e-4


def test_a_short_workspace_is_refused(dev):
    cache, g = build(dev, BF16, 2, 64, 64, 64, [2000], 17)
    q = queries(dev, BF16, 1, 2, 64, g)
    ws = workspace_tensor(omnimem_decode_workspace_bytes(cache, 2), dev)
    with pytest.raises(ValueError, match="workspace holds"):
        omnimem_decode_attn(cache, q, workspace=ws[:-1])
    with pytest.raises(OmniMemError, match="invalid argument"):
        omnimem_decode_attn(cache, q, workspace=torch.empty(ws.numel() + 16, dtype=torch.uint8, device=dev)[16:])
