"""The 8-bit sequence cache's calls together, as a program runs them: prompts and forks and single
tokens over two layers against models of the pages, the step captured into a graph, calls on two
streams at once and on another device than the current one, pools past 32 bits, and attention that
is near the unquantised cache's."""
import random

import pytest
import torch

import quant_oracle
from parity import say
from paper_2605_30519_amd import (SeqKVCache, SeqKVCacheQuant, SeqUpdate, omnimem_append_kv, omnimem_append_kv_quant,
                                  omnimem_copy_pages_quant, omnimem_decode_attn, omnimem_decode_attn_quant,
                                  omnimem_decode_quant_workspace_bytes, omnimem_read_kv_quant, omnimem_seq_compact,
                                  omnimem_seq_update, omnimem_seq_workspace_bytes)
from paper_2605_30519_amd.omnimem import workspace_tensor

pytestmark = pytest.mark.gpu
BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


def i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def check(cache, q, out, lse, B, S):
    O, L, ob, lb = quant_oracle.decode(q, cache.k_pages, cache.v_pages, cache.scales, cache.page_table, cache.seq_lens, B, S, 0,
                                       q.shape[2] ** -0.5)
    assert ((out.double().cpu() - O).abs() <= ob).all()
    full = ~torch.isinf(L)
    assert torch.equal(torch.isinf(lse.cpu()), ~full) and ((lse.double().cpu() - L).abs() <= lb)[full].all()


@pytest.mark.parametrize("dtype,H,G,d,B,S", [(BF16, 2, 3, 128, 64, 64), (F32, 3, 1, 64, 64, 150)])
def test_serving_steps(dev, dtype, H, G, d, B, S):
    """Prompts enter, rows fork, shorten, end and grow, in two layers copied in one call; every page that
    a row holds is the model's code for code, the attention that of those codes, and both stay so
    when the pool is compacted."""
    rng = random.Random(3)
    g = torch.Generator().manual_seed(4)
    layers, P, M = 2, 90, 14
    k, v = (torch.randint(0, 256, (layers, P, H, B, d), generator=g, dtype=torch.uint8) for _ in range(2))
    scales = torch.full((layers, P, H, 2), float("nan"))
    gk, gv, gs = (t.to(dev) for t in (k, v, scales))
    table, lens = torch.zeros((0, M), dtype=torch.int32, device=dev), torch.zeros(0, dtype=torch.int32, device=dev)
    copies = moves = 0

    def same(table, lens):
        for row, t in zip(table.tolist(), lens.tolist()):
            for b in range(M):
                page = row[b]
                n = min(max(t - (b if S == B else b // -(-S // B)) * (B if S == B else S) - (0 if S == B else b % -(-S // B) * B), 0),
                        B if S == B else min(B, S - b % -(-S // B) * B))
                if page >= 0 and n > 0:
                    assert torch.equal(gs[:, page].cpu(), scales[:, page])
                    assert quant_oracle.same_codes(gk[:, page, :, :n], k[:, page, :, :n])
                    assert quant_oracle.same_codes(gv[:, page, :, :n], v[:, page, :, :n])

    for step in range(12):
        parent, keep, grow = [], [], []
        for i, t in enumerate(lens.tolist()):
            for _ in range(rng.choice([0, 1, 1, 1, 2])):
                if len(parent) < 7:
                    parent.append(i)
                    keep.append(rng.choice([t, t, max(0, t - rng.randrange(70))]))
                    grow.append(rng.choice([0, 1, 1, rng.randrange(90)]))
        while len(parent) < 4:
            parent.append(-1)
            keep.append(0)
            grow.append(rng.randrange(1, 200))
        u = omnimem_seq_update(table, lens, P, B, i32(parent, dev), i32(keep, dev), i32(grow, dev), chunk_tokens=S)
        info = u.info.tolist()
        assert info[2:] == [0, 0], (step, info)
        copies += info[0]
        omnimem_copy_pages_quant(gk.view(F8), gv.view(F8), gs, u.copies, u.info)
        for a, b in u.copies.tolist()[:info[0]]:
            for x in (k, v, scales):
                x[:, b] = x[:, a]
        starts = [sum(grow[:i]) for i in range(len(grow) + 1)]
        q = torch.randn((len(parent), H * G, d), generator=g).to(dtype).to(dev)
        before = []
        for layer in range(layers):
            nk, nv = (torch.exp(torch.randn((starts[-1], 1, 1), generator=g)) * torch.randn((starts[-1], H, d), generator=g)
                      for _ in range(2))
            nk, nv = nk.to(dtype), nv.to(dtype)
            cache = SeqKVCacheQuant(gk[layer].view(F8), gv[layer].view(F8), gs[layer], u.page_table, u.seq_lens, S)
            omnimem_append_kv_quant(cache, nk.to(dev), nv.to(dev), i32(starts, dev))
            quant_oracle.append(k[layer], v[layer], scales[layer], u.page_table.tolist(), u.seq_lens.tolist(), nk, nv, starts, S)
            out, lse = omnimem_decode_attn_quant(cache, q)
            check(cache, q, out, lse, B, S)
            before.append((out, lse))
        table, lens = u.page_table, u.seq_lens
        same(table, lens)
        if step % 3 == 2:
            c = omnimem_seq_compact(table, lens, P, B, chunk_tokens=S)
            omnimem_copy_pages_quant(gk.view(F8), gv.view(F8), gs, c.copies, c.info)
            n, used = c.info.tolist()[:2]
            moves += n
            for a, b in c.copies.tolist()[:n]:
                for x in (k, v, scales):
                    x[:, b] = x[:, a]
            for x, y in ((gk, k), (gv, v)):
                x[:, used:] = 0x7f                                # what lies behind is free
                y[:, used:] = 0x7f
            table = c.page_table
            same(table, lens)
            for layer in range(layers):
                cache = SeqKVCacheQuant(gk[layer].view(F8), gv[layer].view(F8), gs[layer], table, lens, S)
                again = omnimem_decode_attn_quant(cache, q)
                assert torch.equal(again[0], before[layer][0]) and torch.equal(again[1], before[layer][1])
    say(f"serving {dtype}: {copies} copies, {moves} moves")
    assert copies > 0 and moves > 0


def test_steps_in_a_graph(dev):
    """Two steps over two sets of buffers, replayed: each replay forks, copies, appends, attends and reads as
    the eager calls do, with lengths that grow from replay to replay."""
    g = torch.Generator(device=dev).manual_seed(9)
    N, H, G, d, B, P, M = 5, 2, 4, 128, 64, 80, 12
    k, v = (torch.randint(0, 120, (P, H, B, d), generator=g, device=dev, dtype=torch.uint8) for _ in range(2))
    scales = torch.exp2(torch.randint(-8, -5, (P, H, 2), generator=g, device=dev).float())
    start = omnimem_seq_update(torch.zeros((0, M), dtype=torch.int32, device=dev),
                               torch.zeros(0, dtype=torch.int32, device=dev), P, B, i32([-1] * N, dev), None,
                               i32([500, 100, 64, 63, 1], dev))
    parent, grow = i32([0, 1, 2, 3, 4], dev), i32([1] * N, dev)
    q = torch.empty((N, H * G, d), dtype=BF16, device=dev)
    nk, nv = torch.empty((N, H, d), dtype=BF16, device=dev), torch.empty((N, H, d), dtype=BF16, device=dev)

    def state():
        sets = [SeqUpdate(start.page_table.clone(), start.seq_lens.clone(), torch.zeros((N, 2), dtype=torch.int32, device=dev),
                          torch.zeros(4, dtype=torch.int32, device=dev)) for _ in range(2)]
        cache = SeqKVCacheQuant(k.clone().view(F8), v.clone().view(F8), scales.clone(), sets[0].page_table, sets[0].seq_lens)
        ws = workspace_tensor(omnimem_decode_quant_workspace_bytes(cache, H * G), dev)
        ts = workspace_tensor(omnimem_seq_workspace_bytes(sets[0].page_table, sets[0].seq_lens, P, B, N), dev)
        out = [torch.empty_like(q) for _ in range(2)] + [torch.empty_like(nk) for _ in range(4)]
        lse = [torch.empty((H * G, N), device=dev) for _ in range(2)]
        return sets, cache, ws, ts, out, lse

    def steps(s):
        sets, cache, ws, ts, out, lse = s
        for a in range(2):
            u = omnimem_seq_update(sets[a].page_table, sets[a].seq_lens, P, B, parent, None, grow, out=sets[1 - a], workspace=ts)
            omnimem_copy_pages_quant(cache.k_pages, cache.v_pages, cache.scales, u.copies, u.info)
            now = cache.after(u)
            omnimem_append_kv_quant(now, nk, nv)
            omnimem_decode_attn_quant(now, q, out=out[a], lse=lse[a], workspace=ws)
            omnimem_read_kv_quant(now, N, out=(out[2 + 2 * a], out[3 + 2 * a]))

    def fill(seed):
        r = torch.Generator(device=dev).manual_seed(seed)
        for t in (q, nk, nv):
            t.copy_(torch.randn(t.shape, generator=r, device=dev) * 2 ** (seed % 4))
        parent.copy_(torch.randint(0, N, (N,), generator=r, device=dev))
        parent[0] = 0

    eager, captured = state(), state()
    fill(0)
    side = torch.cuda.Stream(device=dev)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        steps(state())                # first launches outside the capture
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps(captured)
    torch.cuda.synchronize()
    for rep in range(6):
        say(f"graph replay {rep}")
        fill(rep)
        steps(eager)
        torch.cuda.synchronize()
        for t in captured[4] + captured[5]:
            t.fill_(-9)
        junk = torch.randn(1 << 20, device=dev).sum()      # the program's own eager work
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.isfinite(junk)
        for x, y in zip(eager[0], captured[0]):
            assert torch.equal(x.page_table, y.page_table) and torch.equal(x.seq_lens, y.seq_lens)
            assert torch.equal(x.info, y.info) and torch.equal(x.copies, y.copies) and x.info.tolist()[2:] == [0, 0]
        assert torch.equal(eager[1].k_pages.view(torch.uint8), captured[1].k_pages.view(torch.uint8))
        assert torch.equal(eager[1].v_pages.view(torch.uint8), captured[1].v_pages.view(torch.uint8))
        assert torch.equal(eager[1].scales, captured[1].scales)
        for x, y in zip(eager[4] + eager[5], captured[4] + captured[5]):
            assert torch.equal(x, y)


def made(dev, g, N, t, H, B=64, d=128):
    n = -(-t // B)
    k, v = (torch.randint(0, 120, (N * n, H, B, d), generator=g, device=dev, dtype=torch.uint8) for _ in range(2))
    scales = torch.exp2(torch.randint(-9, -6, (N * n, H, 2), generator=g, device=dev).float())
    return SeqKVCacheQuant(k.view(F8), v.view(F8), scales, torch.randperm(N * n, generator=g, device=dev).int().view(N, n),
                           torch.full((N,), t, dtype=torch.int32, device=dev))


def test_two_graphs_that_share_a_workspace(dev):
    """Nothing in a workspace outlives its call: two graphs over one workspace, replayed in turn."""
    g = torch.Generator(device=dev).manual_seed(21)
    runs = []
    for N, t, H in ((2, 6000, 4), (9, 2500, 2)):
        cache = made(dev, g, N, t, H)
        q = torch.randn((N, 2 * H, 128), generator=g, device=dev).to(BF16)
        runs.append((cache, q, torch.empty_like(q), torch.empty((2 * H, N), device=dev)))
    sizes = [omnimem_decode_quant_workspace_bytes(r[0], r[1].shape[1]) for r in runs]
    assert min(sizes) > 256
    ws = workspace_tensor(max(sizes), dev)
    want = [omnimem_decode_attn_quant(c, q) for c, q, _, _ in runs]
    torch.cuda.synchronize()
    graphs = []
    for cache, q, out, lse in runs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            omnimem_decode_attn_quant(cache, q, out=out, lse=lse, workspace=ws)
    for _ in range(3):
        for graph, r in zip(graphs, runs):
            r[2].fill_(-3)
            graph.replay()
        torch.cuda.synchronize()
        for (o, l), r in zip(want, runs):
            assert torch.equal(r[2], o) and torch.equal(r[3], l)
        for graph in reversed(graphs):
            graph.replay()


def test_two_streams_at_once(dev):
    """Calls on two streams, each with buffers of its own, do not disturb one another."""
    g = torch.Generator(device=dev).manual_seed(11)
    work = [(made(dev, g, N, t, 4), torch.randn((N, 8, 128), generator=g, device=dev).to(dtype))
            for N, t, dtype in ((3, 9000, BF16), (7, 2500, F32))]
    want = [omnimem_decode_attn_quant(*w) + omnimem_read_kv_quant(w[0], w[1].shape[0]) for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(device=dev) for _ in work]
    for _ in range(5):
        got = [[omnimem_decode_attn_quant(*w, stream=s) + omnimem_read_kv_quant(w[0], w[1].shape[0], stream=s.cuda_stream)
                for _ in range(4)] for w, s in zip(work, streams)]
        torch.cuda.synchronize()
        for gs, x in zip(got, want):
            for y in gs:
                assert all(torch.equal(a, b) for a, b in zip(x, y))


def test_appends_and_copies_on_a_stream_of_their_own(dev):
    g = torch.Generator(device=dev).manual_seed(22)
    a = made(dev, g, 4, 300, 3)
    b = SeqKVCacheQuant(a.k_pages.clone(), a.v_pages.clone(), a.scales.clone(), a.page_table, a.seq_lens)
    x = torch.randn((4 * 70, 3, 128), generator=g, device=dev).to(BF16)
    starts = i32([0, 70, 140, 210, 280], dev)
    pairs = i32([[0, 1], [2, 3]], dev)
    torch.cuda.synchronize()
    s = torch.cuda.Stream(device=dev)
    for cache, stream in ((a, None), (b, s)):
        omnimem_append_kv_quant(cache, x, x, starts, stream=stream)
        omnimem_copy_pages_quant(cache.k_pages, cache.v_pages, cache.scales, pairs, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(a.k_pages.view(torch.uint8), b.k_pages.view(torch.uint8))
    assert torch.equal(a.v_pages.view(torch.uint8), b.v_pages.view(torch.uint8)) and torch.equal(a.scales, b.scales)


def test_the_same_call_twice_is_the_same(dev):
    """Bits do not change from call to call, and a repeated append changes nothing."""
    g = torch.Generator(device=dev).manual_seed(23)
    cache = made(dev, g, 11, 1700, 5)
    q = torch.randn((11, 15, 128), generator=g, device=dev).to(BF16)
    a, b = omnimem_decode_attn_quant(cache, q), omnimem_decode_attn_quant(cache, q)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    x = 5 * torch.randn((11 * 33, 5, 128), generator=g, device=dev)
    starts = i32([33 * i for i in range(12)], dev)
    omnimem_append_kv_quant(cache, x, -x, starts)
    was = [t.clone() for t in (cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8), cache.scales)]
    omnimem_append_kv_quant(cache, x, -x, starts)
    for t, w in zip((cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8), cache.scales), was):
        assert torch.equal(t, w)


def test_pools_past_32_bits(dev):
    """Pages whose bytes lie past 2^32: written, copied, attended and read at the pool's end, where a pool of
    few pages gives the same."""
    H, B, d = 8, 64, 128
    P = 2 ** 32 // (H * B * d) + 40                                 # 4.3 GB a pool
    g = torch.Generator(device=dev).manual_seed(12)
    k, v = (torch.empty((P, H, B, d), dtype=torch.uint8, device=dev) for _ in range(2))
    scales = torch.empty((P, H, 2), device=dev)
    n = 30
    T = 2 * n * B - 5
    table = torch.arange(P - 2 * n, P, dtype=torch.int32, device=dev).view(2, n)
    lens, starts = i32([n * B, n * B - 5], dev), i32([0, n * B, T], dev)
    end = SeqKVCacheQuant(k.view(F8), v.view(F8), scales, table, lens)
    fk, fv = (torch.empty((2 * n, H, B, d), dtype=torch.uint8, device=dev) for _ in range(2))
    to = torch.arange(2 * n, dtype=torch.int32, device=dev)
    front = SeqKVCacheQuant(fk.view(F8), fv.view(F8), torch.empty((2 * n, H, 2), device=dev), to.view(2, n), lens)
    nk, nv = (torch.randn((T, H, d), generator=g, device=dev).to(BF16) for _ in range(2))
    q = torch.randn((2, 2 * H, d), generator=g, device=dev).to(BF16)
    got = []
    for cache in (end, front):
        omnimem_append_kv_quant(cache, nk, nv, starts)
        got.append(omnimem_decode_attn_quant(cache, q) + omnimem_read_kv_quant(cache, T, starts))
    check(front, q, got[1][0], got[1][1], B, B)
    assert all(torch.equal(x, y) for x, y in zip(*got))
    assert torch.equal(scales[P - 2 * n:], front.scales)
    # to the pool's front and back again
    omnimem_copy_pages_quant(end.k_pages, end.v_pages, scales, torch.stack([table.flatten(), to], 1).contiguous())
    there = SeqKVCacheQuant(end.k_pages, end.v_pages, scales, to.view(2, n), lens)
    assert all(torch.equal(x, y) for x, y in zip(omnimem_decode_attn_quant(there, q), got[0]))
    k[P - 2 * n:] = 0x7f
    scales[P - 2 * n:] = 3
    omnimem_copy_pages_quant(end.k_pages, end.v_pages, scales, torch.stack([to, table.flatten()], 1).contiguous())
    assert all(torch.equal(x, y) for x, y in zip(omnimem_decode_attn_quant(end, q), got[0]))


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
def test_attention_is_near_the_unquantised_caches(dev, dtype, d):
    """Keys and values off by 2^-4 of themselves at most leave attention off by what that does to scores
    and values: |ds| <= 2^-4 scale sum |q k|, the outputs by (e^{2 |ds|} - 1 + 2^-4) of the values' spread."""
    g = torch.Generator(device=dev).manual_seed(30)
    N, H, G, t, B = 3, 2, 4, 700, 64
    n = -(-t // B)
    table = torch.randperm(N * n, generator=g, device=dev).int().view(N, n)
    lens = i32([t] * N, dev)
    nk, nv = (torch.randn((N * t, H, d), generator=g, device=dev).to(dtype) for _ in range(2))
    q = (0.3 * torch.randn((N, H * G, d), generator=g, device=dev)).to(dtype)
    plain = SeqKVCache(*(torch.zeros((N * n, H, B, d), dtype=dtype, device=dev) for _ in range(2)), table, lens)
    quant = SeqKVCacheQuant(*(torch.zeros((N * n, H, B, d), dtype=torch.uint8, device=dev).view(F8) for _ in range(2)),
                            torch.zeros((N * n, H, 2), device=dev), table, lens)
    starts = i32([t * i for i in range(N + 1)], dev)
    omnimem_append_kv(plain, nk, nv, starts)
    omnimem_append_kv_quant(quant, nk, nv, starts)
    a, b = omnimem_decode_attn(plain, q), omnimem_decode_attn_quant(quant, q)
    kk, qq, vv = nk.double().view(N, t, H, d), q.double().view(N, H, G, d), nv.double().view(N, t, H, d)
    ds = 2.0 ** -4 * d ** -0.5 * torch.einsum("nthd,nhgd->nhgt", kk.abs().cpu(), qq.abs().cpu()).amax(-1)
    assert ((a[1] - b[1]).double().cpu().t().reshape(N, H, G).abs() <= ds + 1e-4).all()
    spread = vv.abs().cpu().amax(1)[:, :, None]                       # a weighted mean of |v| is no more
    bound = (torch.exp(2 * ds)[..., None] - 1 + 2.0 ** -4) * spread + 2.0 ** -7 * spread
    assert ((a[0] - b[0]).double().cpu().view(N, H, G, d).abs() <= bound).all()
    # and the mean error is that of rounding: far below the bound
    rms = (a[0] - b[0]).float().square().mean().sqrt() / a[0].float().square().mean().sqrt()
    assert rms < 2.0 ** -4
