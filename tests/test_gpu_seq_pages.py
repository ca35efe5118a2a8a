"""The sequence cache's pages: omnimem_append_kv, omnimem_copy_pages, omnimem_seq_update and
omnimem_seq_compact against list models, whole pools compared bit for bit."""
import random

import pytest
import torch

import seq_oracle
from parity import say
from paper_2605_30519_amd import (SeqKVCache, SeqUpdate, omnimem_append_kv, omnimem_copy_pages, omnimem_seq_compact,
                                  omnimem_seq_update, omnimem_seq_workspace_bytes)
from paper_2605_30519_amd.omnimem import workspace_tensor

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


def i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


# ------------------------------------------------------------------------- append


def append_case(dev, dtype, H, d, B, S, lens, new, seed, extra_blocks=0, drop=(), ragged=True, stride=1):
    g = torch.Generator().manual_seed(seed)
    nb = [seq_oracle.blocks(t, S, B) for t in lens]
    M, P = max(nb + [1]) + extra_blocks, sum(nb) + 2
    ids = torch.randperm(P, generator=g).tolist()
    table = [[ids.pop() for _ in range(n)] + [-1] * (M - n) for n in nb]
    for i, b, page in drop:
        table[i][b] = page
    k = torch.randn((P, H, B, d), generator=g).to(dtype)
    v = torch.randn((P, H, B, d), generator=g).to(dtype)
    T = sum(new)
    nk = torch.randn((T, stride, H, d), generator=g).to(dtype)
    nv = torch.randn((T, stride, H, d), generator=g).to(dtype)
    want_k, want_v, row = k.clone(), v.clone(), 0
    cap = seq_oracle.capacity(M, S, B)
    for i, (t, n) in enumerate(zip(lens, new)):
        for x in range(t - n, t):
            if 0 <= x < cap:
                b, s = seq_oracle.place(x, S, B)
                if 0 <= table[i][b] < P:
                    want_k[table[i][b], :, s] = nk[row, 0]
                    want_v[table[i][b], :, s] = nv[row, 0]
            row += 1
    cache = SeqKVCache(k.to(dev), v.to(dev), i32(table, dev).view(len(lens), M), i32(lens, dev), S)
    starts = None
    if ragged:
        starts = i32([sum(new[:i]) for i in range(len(new) + 1)], dev)
    omnimem_append_kv(cache, nk.to(dev)[:, 0], nv.to(dev)[:, 0], starts)
    torch.cuda.synchronize()
    assert torch.equal(cache.k_pages.cpu(), want_k) and torch.equal(cache.v_pages.cpu(), want_v)


@pytest.mark.parametrize("dtype,H,d", [(BF16, 1, 64), (BF16, 12, 128), (F32, 3, 64), (F32, 40, 128)])
@pytest.mark.parametrize("B,S", [(64, 64), (128, 128), (64, 100), (128, 300)])
def test_append_ragged(dev, dtype, H, d, B, S):
    say(f"append {dtype} H={H} d={d} B={B} S={S}")
    append_case(dev, dtype, H, d, B, S, [5, 130, 64, 0, 301, 65], [5, 70, 1, 0, 300, 2], 1)


@pytest.mark.parametrize("dtype,H,d", [(BF16, 1, 64), (BF16, 8, 128), (F32, 5, 128)])
def test_append_one_token_each(dev, dtype, H, d):
    lens = [1, 2, 64, 65, 128, 129, 700] * 11
    append_case(dev, dtype, H, d, 64, 64, lens, [1] * len(lens), 2, ragged=False)
    append_case(dev, dtype, H, d, 64, 64, lens, [1] * len(lens), 3, stride=3)


def test_append_long(dev):
    append_case(dev, BF16, 2, 64, 64, 64, [20000, 3], [20000, 1], 4)
    append_case(dev, BF16, 12, 128, 64, 4680, [9360, 4680], [4680, 4680], 5)


def test_append_drops_what_has_no_place(dev):
    # more new tokens than the sequence has; a block that is not resident, one with no such page
    append_case(dev, BF16, 2, 64, 64, 64, [10, 200, 200], [30, 200, 150], 6, drop=[(1, 1, -1), (2, 2, 1 << 20)])


def test_append_past_the_capacity_and_odd_starts(dev):
    cache = SeqKVCache(torch.zeros((4, 1, 64, 64), device=dev), torch.zeros((4, 1, 64, 64), device=dev),
                       i32([[0, 1], [2, 3]], dev), i32([150, -4], dev))
    k = torch.arange(1, 31, device=dev, dtype=F32)[:, None, None].expand(30, 1, 64).contiguous()
    omnimem_append_kv(cache, k, -k, i32([0, 30, 30], dev))
    got = cache.k_pages[:2, 0, :, 0].flatten()
    # token 120 + r is row r: rows 0 .. 7 fit under the capacity of 128
    assert torch.equal(got[120:], torch.arange(1, 9, device=dev, dtype=F32)) and got[:120].eq(0).all()
    assert cache.k_pages[2:].eq(0).all()
    cache.seq_lens.copy_(i32([64, 100], dev))
    cache.k_pages.zero_()
    omnimem_append_kv(cache, k, k, i32([-5, 10, 99], dev))     # clamped to [0, 10) and [10, 30)
    assert torch.equal(cache.k_pages[0, 0, 54:, 0], k[:10, 0, 0])
    assert torch.equal(cache.k_pages[2:, 0, :, 0].flatten()[80:100], k[10:, 0, 0])
    assert int(cache.k_pages[..., 0].ne(0).sum()) == 30


def test_append_to_more_sequences_than_threads(dev):
    lens = [1 + i % 70 for i in range(600)]
    append_case(dev, F32, 1, 64, 64, 64, lens, [(i * 7) % (t + 1) for i, t in enumerate(lens)], 7)


def test_append_leaves_rows_behind_the_last_start(dev):
    cache = SeqKVCache(torch.zeros((4, 2, 64, 64), device=dev), torch.zeros((4, 2, 64, 64), device=dev),
                       i32([[0, 1], [2, 3]], dev), i32([70, 3], dev))
    k = torch.ones((50, 2, 64), device=dev)
    omnimem_append_kv(cache, k, k, i32([2, 10, 12], dev))
    assert int(cache.k_pages[..., 0].sum()) == 2 * (8 + 2)
    assert cache.k_pages[0, :, 62:].eq(1).all() and cache.k_pages[1, :, :6].eq(1).all() and cache.k_pages[2, :, 1:3].eq(1).all()


def test_append_nothing(dev):
    append_case(dev, BF16, 2, 64, 64, 64, [10, 0], [0, 0], 8)
    append_case(dev, BF16, 2, 64, 64, 64, [], [], 9)


# ------------------------------------------------------------------------- copies


@pytest.mark.parametrize("dtype,shape,layers", [(BF16, (40, 1, 64, 64), 0), (F32, (17, 5, 128, 128), 0),
                                                (BF16, (30, 12, 64, 128), 3), (torch.uint8, (9, 1, 3, 16), 2),
                                                (BF16, (500, 1, 64, 64), 1)])
def test_copy_pages(dev, dtype, shape, layers):
    say(f"copy {dtype} {shape} layers={layers}")
    g = torch.Generator().manual_seed(1)
    full = ((layers,) if layers else ()) + shape
    k = torch.randint(0, 100, full, generator=g).to(dtype)
    v = torch.randint(0, 100, full, generator=g).to(dtype)
    P = shape[0]
    ids = torch.randperm(P, generator=g).tolist()
    n = P // 2
    pairs = [(ids[n + i % (P - n) // 2], ids[i]) for i in range(n)] + [(-1, ids[0]), (ids[-1], P), (P + 5, ids[1]), (ids[-1], -7)]
    for count in (None, 0, 1, n, len(pairs), 10 ** 6, -1):
        m = len(pairs) if count is None else min(max(count, 0), len(pairs))
        want_k, want_v = k.clone(), v.clone()
        for s, t in pairs[:m]:
            if 0 <= s < P and 0 <= t < P:
                (want_k[:, t] if layers else want_k[t]).copy_(k[:, s] if layers else k[s])
                (want_v[:, t] if layers else want_v[t]).copy_(v[:, s] if layers else v[s])
        gk, gv = k.to(dev), v.to(dev)
        omnimem_copy_pages(gk, gv, i32(pairs, dev), None if count is None else i32([count, 7], dev))
        torch.cuda.synchronize()
        assert torch.equal(gk.cpu(), want_k) and torch.equal(gv.cpu(), want_v)
    gk = k.to(dev)
    omnimem_copy_pages(gk, None, i32(pairs, dev))
    want_k = k.clone()
    for s, t in pairs[:n]:
        (want_k[:, t] if layers else want_k[t]).copy_(k[:, s] if layers else k[s])
    assert torch.equal(gk.cpu(), want_k)


def test_copy_layers_apart(dev):
    """Layers of a larger allocation, with other tensors between them."""
    both = torch.randint(0, 100, (3, 2, 6, 2, 64, 64), device=dev).to(BF16)
    k, v = both[:, 0], both[:, 1]
    want = both.clone()
    want[:, :, 5] = both[:, :, 2]
    omnimem_copy_pages(k, v, i32([[2, 5]], dev))
    assert torch.equal(both, want)


# ------------------------------------------------------------------------- tables


def update_and_check(dev, table, lens, P, B, S, parent, keep, grow, **kw):
    args = [None if x is None else i32(x, dev) for x in (parent, keep, grow)]
    M = len(table[0]) if table else 3
    t, l = i32(table, dev).view(len(table), M), i32(lens, dev)
    u = omnimem_seq_update(t, l, P, B, *args, chunk_tokens=S, **kw)
    torch.cuda.synchronize()
    rows, want_lens, copies, info = seq_oracle.update(table or [[-1] * M], lens or [0], P, B, S or B,
                                                      parent if table else [-1] * len(parent), keep, grow)
    assert u.info.tolist() == info
    assert u.seq_lens.tolist() == want_lens
    assert u.page_table.tolist() == rows
    assert u.copies.tolist() == [list(c) for c in copies] + [[-1, -1]] * (len(parent) - len(copies))
    assert t.tolist() == table and l.tolist() == lens
    return u


def random_tables(rng, N, P, B, S, most, share=0.5, bad=0.1):
    ids = list(range(P))
    rng.shuffle(ids)
    table, lens = [], []
    for i in range(N):
        t = rng.choice([0, rng.randrange(most + 1), rng.randrange(most + 1)])
        n = seq_oracle.blocks(t, S, B)
        row = [ids.pop() if ids else -1 for _ in range(n)]
        if i and rng.random() < share:
            j = rng.randrange(i)
            m = rng.randrange(min(n, len(table[j])) + 1)
            row[:m] = table[j][:m]
        for b in range(n):
            if rng.random() < bad / max(n, 1):
                row[b] = rng.choice([-1, P, -2 ** 31, 2 ** 31 - 1])
        table.append(row)
        lens.append(t)
    return table, lens


@pytest.mark.parametrize("B,S", [(64, 0), (128, 0), (64, 100), (128, 700), (64, 10)])
@pytest.mark.parametrize("seed", range(6))
def test_update_random(dev, B, S, seed):
    rng = random.Random(f"{B} {S} {seed}")
    done = grown = copied = 0
    for _ in range(8):
        N, P = rng.randrange(1, 40), rng.choice([1, 31, 32, 33, 200, 1000])
        most = rng.choice([70, 500, 1500])
        table, lens = random_tables(rng, N, P, B, S or B, most)
        M = max([len(r) for r in table] + [1]) + rng.randrange(3)
        table = [r + [rng.choice([-1, 5])] * (M - len(r)) for r in table]
        R = rng.randrange(1, 50)
        parent = [rng.choice([rng.randrange(N), rng.randrange(N), min(i, N - 1), -1, N, 2 ** 31 - 1]) for i in range(R)]
        keep = rng.choice([None, [rng.choice([10 ** 9, -3, rng.randrange(most + 1)]) for _ in range(R)]])
        grow = rng.choice([None, [rng.choice([0, 1, 1, -2, rng.randrange(200)]) for _ in range(R)]])
        u = update_and_check(dev, table, lens, P, B, S, parent, keep, grow)
        info = u.info.tolist()
        done += 1
        grown += info[2] == info[3] == 0
        copied += info[0]
    say(f"update B={B} S={S} seed={seed}: {done} calls, {grown} with room, {copied} copies")


def test_update_beam_step(dev):
    """Two children of one row: the lower keeps the begun page, the other copies it."""
    u = update_and_check(dev, [[3, 1], [0, 4]], [100, 70], 8, 64, 0, [0, 0, 1], None, [1, 1, 1])
    assert u.page_table.tolist() == [[3, 1], [3, 2], [0, 4]] and u.copies.tolist()[0] == [1, 2]
    # a third row that holds the page and does not grow: both growing rows copy
    u = update_and_check(dev, [[3, 1], [0, 4]], [100, 70], 9, 64, 0, [0, 0, 0], None, [1, 0, 1])
    assert u.info.tolist()[0] == 2
    # a shorter fork of a full block still begins a copy
    u = update_and_check(dev, [[3, 1, -1]], [128], 9, 64, 0, [0, 0], [128, 70], [1, 1])
    assert u.copies.tolist()[0] == [1, 2] and u.page_table.tolist() == [[3, 1, 0], [3, 2, -1]]


def test_update_with_a_page_twice_in_a_row(dev):
    u = update_and_check(dev, [[3, 3, 5]], [150], 8, 64, 0, [0], None, [1])
    assert u.copies.tolist() == [[-1, -1]]
    u = update_and_check(dev, [[3, 5, 3]], [150], 8, 64, 0, [0, 0], [150, 140], [1, 64])
    assert u.info.tolist() == [0, 2, 0, 1]                          # 204 tokens in a row of 192
    u = update_and_check(dev, [[3, 5, 3]], [150], 8, 64, 0, [0, 0], [150, 140], [1, 52])
    assert u.info.tolist() == [2, 4, 0, 0]                          # page 3 is a full block too
    compact_and_check(dev, [[7, 6, 7], [6, 6, 6]], [150, 129], 8, 64, 0)


def test_update_frees_and_takes_the_lowest_pages(dev):
    u = update_and_check(dev, [[7, 2], [5, 6]], [128, 128], 8, 64, 0, [1, -1], None, [0, 100])
    assert u.page_table.tolist() == [[5, 6], [0, 1]]
    u = update_and_check(dev, [[7, 2], [5, 6]], [128, 128], 8, 64, 0, [], None, None)
    assert u.info.tolist() == [0, 0, 0, 0]


def test_update_short_of_pages_or_capacity(dev):
    table, lens = [[0, 1, -1, -1], [2, -1, -1, -1]], [128, 30]
    u = update_and_check(dev, table, lens, 4, 64, 0, [0, 1], None, [64, 40])     # one more page than there is
    assert u.info.tolist() == [0, 3, 1, 0] and u.seq_lens.tolist() == [128, 30]
    u = update_and_check(dev, table, lens, 9, 64, 0, [0, 1], None, [129, 1])     # one token past a row
    assert u.info.tolist() == [0, 3, 0, 1] and u.seq_lens.tolist() == [128, 30]
    u = update_and_check(dev, table, lens, 9, 64, 0, [0, 1], None, [128, 2 ** 31 - 1])
    assert u.info.tolist() == [0, 3, 0, 1]
    u = update_and_check(dev, table, lens, 9, 64, 0, [0, 1], None, [128, 226])   # every row full
    assert u.info.tolist() == [0, 8, 0, 0]


def test_update_lengths_out_of_range(dev):
    update_and_check(dev, [[0, 1], [2, 3]], [2 ** 31 - 1, -5], 9, 64, 0, [0, 1, 1], None, [0, 3, 0])


def test_update_without_pages_or_rows(dev):
    update_and_check(dev, [[0, 1]], [70], 0, 64, 0, [0], None, [0])
    update_and_check(dev, [[0, 1]], [70], 0, 64, 0, [0], None, [60])
    update_and_check(dev, [], [], 50, 64, 0, [-1, 4], None, [1, 130])


def test_update_large(dev):
    """More rows than threads of a workgroup, more pages than 32 a thread."""
    rng = random.Random(4)
    table, lens = random_tables(rng, 1300, 40000, 64, 64, 1500)
    M = max(len(r) for r in table) + 1
    table = [r + [-1] * (M - len(r)) for r in table]
    parent = [rng.randrange(1300) if rng.random() < 0.3 else i for i in range(1400)]
    u = update_and_check(dev, table, lens, 40000, 64, 0, parent, None, [rng.randrange(100) for _ in parent])
    assert u.info.tolist()[0] > 50 and u.info.tolist()[2:] == [0, 0]


def compact_and_check(dev, table, lens, P, B, S):
    M = len(table[0]) if table else 2
    t, l = i32(table, dev).view(len(table), M), i32(lens, dev)
    u = omnimem_seq_compact(t, l, P, B, chunk_tokens=S)
    rows, moves, info = seq_oracle.compact(table, lens, P, B, S or B)
    assert u.info.tolist() == info and u.page_table.tolist() == rows
    assert u.copies.tolist() == [list(m) for m in moves] + [[-1, -1]] * (max(1, P // 2) - len(moves))
    assert u.seq_lens is l
    return u


@pytest.mark.parametrize("B,S", [(64, 0), (128, 0), (64, 100), (128, 700)])
@pytest.mark.parametrize("seed", range(4))
def test_compact_random(dev, B, S, seed):
    rng = random.Random(f"compact {B} {S} {seed}")
    moved = 0
    for _ in range(8):
        N, P = rng.randrange(1, 40), rng.choice([1, 2, 31, 32, 33, 64, 300, 2000])
        table, lens = random_tables(rng, N, P, B, S or B, rng.choice([70, 600]))
        M = max([len(r) for r in table] + [1])
        moved += compact_and_check(dev, [r + [0] * (M - len(r)) for r in table], lens, P, B, S).info.tolist()[0]
    say(f"compact B={B} S={S} seed={seed}: {moved} moves")


def test_compact_edges(dev):
    compact_and_check(dev, [[0, 1]], [100], 2, 64, 0)              # a full pool
    compact_and_check(dev, [[1, 9]], [0], 2, 64, 0)                # nothing in use
    compact_and_check(dev, [[5, 9]], [100], 0, 64, 0)              # no pages
    compact_and_check(dev, [], [], 70, 64, 0)                      # no rows
    compact_and_check(dev, [[39, 38, 37, 0]], [256], 40, 64, 0)
    rng = random.Random(9)
    table, lens = random_tables(rng, 900, 50000, 64, 64, 1500)
    M = max(len(r) for r in table)
    u = compact_and_check(dev, [r + [-1] * (M - len(r)) for r in table], lens, 50000, 64, 0)
    assert u.info.tolist()[0] > 1000


def test_a_dirty_workspace(dev):
    """Tables past one workgroup's, with scratch that another use has left full."""
    rng = random.Random(6)
    table, lens = random_tables(rng, 300, 17000, 64, 64, 1500)
    M = max(len(r) for r in table) + 1
    table = [r + [-1] * (M - len(r)) for r in table]
    t, l = i32(table, dev), i32(lens, dev)
    need = omnimem_seq_workspace_bytes(t, l, 17000, 64, 300)
    assert need > 256
    for fill in (255, 0, 127):
        ws = workspace_tensor(need, dev).fill_(fill)
        update_and_check(dev, table, lens, 17000, 64, 0, list(range(300)), None, [1] * 300, workspace=ws)
        ws.fill_(fill)
        c = omnimem_seq_compact(t, l, 17000, 64, workspace=ws)
        rows, _, info = seq_oracle.compact(table, lens, 17000, 64, 64)
        assert c.info.tolist() == info and c.page_table.tolist() == rows


def test_given_buffers_and_workspace(dev):
    t, l = i32([[3, 1], [0, 4]], dev), i32([100, 70], dev)
    ws = workspace_tensor(omnimem_seq_workspace_bytes(t, l, 8, 64, 2), dev)
    ws.fill_(255)
    out = SeqUpdate(torch.full_like(t, 77), torch.full_like(l, 77), i32([[9, 9], [9, 9]], dev), i32([9] * 4, dev))
    u = omnimem_seq_update(t, l, 8, 64, i32([0, 0], dev), None, i32([1, 1], dev), out=out, workspace=ws)
    assert u is out and u.page_table.tolist() == [[3, 1], [3, 0]] and u.copies.tolist() == [[1, 0], [-1, -1]]
    assert u.info.tolist() == [1, 3, 0, 0] and u.seq_lens.tolist() == [101, 101]
    side = torch.cuda.Stream(device=dev)
    side.wait_stream(torch.cuda.current_stream())
    u2 = omnimem_seq_update(t, l, 8, 64, i32([0, 0], dev), None, i32([1, 1], dev), stream=side)
    torch.cuda.synchronize()
    assert torch.equal(u2.page_table, u.page_table)
    c = omnimem_seq_compact(t, l, 8, 64, stream=side)
    torch.cuda.synchronize()
    assert c.page_table.tolist() == [[3, 1], [0, 2]] and c.copies.tolist()[0] == [4, 2]
