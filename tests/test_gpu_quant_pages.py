"""omnimem_append_kv_quant, omnimem_read_kv_quant and omnimem_copy_pages_quant against models on the CPU: every
code and scale of the pools equal, what a call does not write left as it was."""
import random

import pytest
import torch

import quant_oracle
import seq_oracle
from parity import say
from paper_2605_30519_amd import (SeqKVCacheQuant, omnimem_append_kv_quant, omnimem_copy_pages_quant,
                                  omnimem_read_kv_quant)

pytestmark = pytest.mark.gpu
BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


def i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def pools(P, H, B, d, g, low=-12, high=2):
    """Random codes, NaN among them, and power-of-two scales, on the CPU."""
    k, v = (torch.randint(0, 256, (P, H, B, d), generator=g, dtype=torch.uint8) for _ in range(2))
    return k, v, torch.exp2(torch.randint(low, high, (P, H, 2), generator=g).float())


def tables(lens, S, B, g, extra_blocks=1, spare=2):
    nb = [seq_oracle.blocks(max(t, 0), S, B) for t in lens]
    M = max(nb) + extra_blocks
    P = sum(nb) + spare
    ids = torch.randperm(P, generator=g).tolist()
    return [[ids.pop() for _ in range(n)] + [-1] * (M - n) for n in nb], P


def append_and_compare(dev, k, v, scales, table, lens, nk, nv, starts, S, B):
    gk, gv, gs = k.to(dev), v.to(dev), scales.to(dev)
    cache = SeqKVCacheQuant(gk.view(F8), gv.view(F8), gs, i32(table, dev), i32(lens, dev), S)
    omnimem_append_kv_quant(cache, nk.to(dev), nv.to(dev), None if starts is None else i32(starts, dev))
    torch.cuda.synchronize()
    quant_oracle.append(k, v, scales, table, lens, nk, nv, starts, S)
    assert torch.equal(gs.cpu().nan_to_num(-1), scales.nan_to_num(-1)), "scales"
    assert quant_oracle.same_codes(gk, k), "K"
    assert quant_oracle.same_codes(gv, v), "V"
    return cache


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,B,H", [(128, 64, 3), (64, 64, 2), (128, 128, 1), (64, 128, 5)])
@pytest.mark.parametrize("S", [0, 100, 300])
def test_appends_of_every_length(dev, dtype, d, B, H, S):
    say(f"append {dtype} d={d} B={B} H={H} S={S}")
    S = S or B
    g = torch.Generator().manual_seed(d + B + S)
    lens = [1, 5, 64, 65, 127, 128, 129, 200, 300, 420, 64, 33]
    new = [1, 2, 64, 1, 63, 64, 129, 0, 300, 133, 1, 20]
    table, P = tables(lens, S, B, g)
    k, v, scales = pools(P, H, B, d, g)
    T = sum(new) + 3                                         # rows of no sequence behind the last
    size = torch.exp(1.5 * torch.randn((T, H, 1), generator=g))
    nk, nv = ((size * torch.randn((T, H, d), generator=g)).to(dtype) for _ in range(2))
    starts = [sum(new[:i]) for i in range(len(new) + 1)]
    append_and_compare(dev, k, v, scales, table, lens, nk, nv, starts, S, B)


@pytest.mark.parametrize("dtype,d,B", [(BF16, 128, 64), (F32, 64, 128)])
def test_one_token_each(dev, dtype, d, B):
    g = torch.Generator().manual_seed(5)
    lens = [1, 2, 64, 65, 66, 128, 129, 500, 0, -4, 1000]
    table, P = tables(lens, B, B, g)
    k, v, scales = pools(P, 4, B, d, g)
    size = torch.exp(2 * torch.randn((len(lens), 4, 1), generator=g))
    nk, nv = ((size * torch.randn((len(lens), 4, d), generator=g)).to(dtype) for _ in range(2))
    append_and_compare(dev, k, v, scales, table, lens, nk, nv, None, B, B)


def test_values_at_the_ends_of_their_type(dev):
    """Zeros, subnormals, the largest numbers, infinities and NaN; scales as they must not be."""
    g = torch.Generator().manual_seed(6)
    big = torch.finfo(F32).max
    special = [0.0, -0.0, 2.0 ** -149, 2.0 ** -126, 2.0 ** -120, 1.75 * 2.0 ** -102, 448.0, 448.0001, 1.75, 1.7500001, big, -big,
               2.0 ** 127, float("inf"), -float("inf"), float("nan"), 1e-30, 3e30]
    lens = [64] * len(special) + [40] * len(special)
    new = [64] * len(special) + [3] * len(special)
    table, P = tables(lens, 64, 64, g)
    k, v, scales = pools(P, 2, 64, 64, g, -120, 125)
    odd = torch.tensor([0.0, -1.0, float("inf"), float("nan"), 1e-45, 3.0, 1.5 * 2.0 ** 100, 2.0 ** 127, 2.0 ** -126, 2.0 ** 120])
    scales.view(-1)[:] = torch.where(torch.rand(scales.numel(), generator=g) < 0.4, odd[torch.arange(scales.numel()) % 10],
                                     scales.view(-1))
    T = sum(new)
    nk = torch.randn((T, 2, 64), generator=g) * 1e-3
    nv = nk * 2.0 ** -110
    at = 0
    for x, n in zip(special * 2, new):
        nk[at + n // 2, 0, 7] = x
        nv[at, 1, 63] = x
        at += n
    starts = [sum(new[:i]) for i in range(len(new) + 1)]
    for dtype in (F32, BF16):
        append_and_compare(dev, k.clone(), v.clone(), scales.clone(), table, lens, nk.to(dtype), nv.to(dtype), starts, 64, 64)


def test_rows_without_a_place(dev):
    """More rows than the sequence has tokens, tokens behind the capacity, blocks that are not resident,
    starts out of range, no rows: what has no place is dropped, the rest of the pool stays."""
    g = torch.Generator().manual_seed(7)
    lens = [10, 400, 200, -5, 2 ** 31 - 1, 70, 300]
    table = [[0, -1, -1, -1], [1, 2, 3, 4], [5, -1, 9999, 6], [7, 8, -1, -1], [9, 10, 11, 12], [13, 14, -1, -1], [15, 16, 17, 18]]
    k, v, scales = pools(20, 3, 64, 128, g)
    new = [30, 250, 200, 4, 9, 0, 60]
    T = sum(new) - 20
    nk, nv = (torch.randn((T, 3, 128), generator=g).to(BF16) for _ in range(2))
    starts = [sum(new[:i]) for i in range(len(new) + 1)]          # the last ones lie behind T
    starts[0] = -7
    append_and_compare(dev, k, v, scales, table, lens, nk, nv, starts, 64, 64)
    # S = 100: the capacity of four blocks is 200 tokens
    append_and_compare(dev, k, v, scales, table, [120, 201, 100, 0, 250, 199, 200], nk, nv, starts, 100, 64)


def test_strided_rows(dev):
    g = torch.Generator().manual_seed(8)
    lens, new = [100, 64], [70, 3]
    table, P = tables(lens, 64, 64, g)
    k, v, scales = pools(P, 2, 64, 128, g)
    for dtype in (BF16, F32):
        fused = torch.randn((73, 4, 2, 128), generator=g).to(dtype)
        gk, gv, gs = k.to(dev), v.to(dev), scales.to(dev)
        f = fused.to(dev)
        omnimem_append_kv_quant(SeqKVCacheQuant(gk.view(F8), gv.view(F8), gs, i32(table, dev), i32(lens, dev)), f[:, 1], f[:, 3],
                                i32([0, 70, 73], dev))
        wk, wv, ws = k.clone(), v.clone(), scales.clone()
        quant_oracle.append(wk, wv, ws, table, lens, fused[:, 1], fused[:, 3], [0, 70, 73], 64)
        assert quant_oracle.same_codes(gk, wk) and quant_oracle.same_codes(gv, wv) and torch.equal(gs.cpu(), ws)


@pytest.mark.parametrize("pieces", [[1] * 90, [7] * 12 + [6], [64, 26], [63, 2, 25]])
def test_in_how_many_calls_hardly_matters(dev, pieces):
    """The scales are those of one append, and so are all values but those below 2^-6 of their scale,
    which are rounded again each time the scale doubles: 1/2 + 1/4 + 1/8 .. of e4m3's smallest step and the
    half step of one append, less than two steps, so that what are whole steps differ by one at most."""
    g = torch.Generator().manual_seed(9)
    size = torch.exp(torch.linspace(-4, 2, 90))[:, None, None] * torch.exp(torch.randn((90, 2, 1), generator=g))
    x = (size * torch.randn((90, 2, 128), generator=g)).to(BF16).to(dev)
    table = i32([[0, 1]], dev)

    def fill(pieces):
        k, v = (torch.full((2, 2, 64, 128), 0x55, dtype=torch.uint8, device=dev) for _ in range(2))
        scales = torch.full((2, 2, 2), 2.0 ** 60, device=dev)     # of nothing: a block's first token sets its own
        at = 0
        for n in pieces:
            omnimem_append_kv_quant(SeqKVCacheQuant(k.view(F8), v.view(F8), scales, table, i32([at + n], dev)), x[at:at + n],
                                    x[at:at + n], i32([0, n], dev))
            at += n
        assert torch.equal(k, v)
        return k.view(F8).float(), scales

    (a, sa), (b, sb) = fill([90]), fill(pieces)
    assert torch.equal(sa, sb) and float(sa.max()) < 1
    small = a.abs() < 2.0 ** -6
    assert torch.equal(a[~small & (b.abs() >= 2.0 ** -6)], b[~small & (b.abs() >= 2.0 ** -6)])
    assert (a - b).abs().max() <= 2.0 ** -9
    if pieces == [64, 26]:                                       # whole blocks: nothing is rounded twice
        assert torch.equal(a, b)


def test_many_sequences(dev):
    """Numbers of sequences around and far past a wave's lanes, most of them without a page."""
    g = torch.Generator().manual_seed(10)
    for N in (63, 64, 65, 4096, 4097, 9000):
        say(f"append to {N} sequences")
        new = torch.randint(0, 3, (N,), generator=g)
        new[5] = 200
        lens = (new + torch.randint(0, 150, (N,), generator=g)).clamp(max=255)
        table = torch.full((N, 4), -1, dtype=torch.int32)
        some = sorted({0, 1, 5, N // 2, N - 2, N - 1})
        for j, i in enumerate(some):
            table[i] = torch.arange(4 * j, 4 * j + 4)
        k, v, scales = pools(4 * len(some), 1, 64, 64, g)
        starts = torch.cat([torch.zeros(1, dtype=torch.long), new.cumsum(0)])
        nk, nv = (torch.randn((int(starts[-1]), 1, 64), generator=g) for _ in range(2))
        append_and_compare(dev, k, v, scales, table.tolist(), lens.tolist(), nk, nv, starts.tolist(), 64, 64)


def test_more_work_than_workgroups(dev):
    """Over 2^22 (block, head, pool) triples: workgroups take further ones in turn."""
    N, H, d = 140000, 16, 64
    g = torch.Generator(device=dev).manual_seed(11)
    table = torch.full((N, 1), -1, dtype=torch.int32, device=dev)
    some = torch.tensor([0, 7, N // 2, N - 3, N - 1], device=dev)
    table[some, 0] = torch.arange(5, dtype=torch.int32, device=dev)
    x = torch.randn((N, H, d), generator=g, device=dev).to(BF16)
    k, v = (torch.zeros((5, H, 64, d), dtype=torch.uint8, device=dev) for _ in range(2))
    scales = torch.zeros((5, H, 2), device=dev)
    omnimem_append_kv_quant(SeqKVCacheQuant(k.view(F8), v.view(F8), scales, table, torch.ones(N, dtype=torch.int32, device=dev)), x, x)
    torch.cuda.synchronize()
    wk, wv, ws = (torch.zeros_like(t).cpu() for t in (k, v, scales))
    quant_oracle.append(wk, wv, ws, [[i] for i in range(5)], [1] * 5, x[some].cpu(), x[some].cpu(), None, 64)
    assert quant_oracle.same_codes(k, wk) and quant_oracle.same_codes(v, wv) and torch.equal(scales.cpu(), ws)


# ------------------------------------------------------------------------- read

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,B,H,S", [(128, 64, 3, 64), (64, 64, 1, 100), (128, 128, 2, 300), (64, 128, 5, 128)])
def test_tokens_read_back(dev, dtype, d, B, H, S):
    say(f"read {dtype} d={d} B={B} H={H} S={S}")
    g = torch.Generator().manual_seed(12)
    lens = [1, 64, 65, 300, 0, -3, 200, 2 ** 31 - 1, 150]
    table, P = tables([1, 64, 65, 300, 0, 0, 200, 250, 150], S, B, g, extra_blocks=0)
    table[6][1] = -1
    table[8][0] = P
    k, v, scales = pools(P, H, B, d, g)
    scales *= 1 + torch.rand(scales.shape, generator=g)          # any scale
    n = [1, 70, 3, 300, 2, 5, 200, 9, 0]
    T = sum(n) + 4
    starts = [sum(n[:i]) for i in range(len(n) + 1)]
    cache = SeqKVCacheQuant(k.to(dev).view(F8), v.to(dev).view(F8), scales.to(dev), i32(table, dev), i32(lens, dev), S)
    for first in (None, [0, -2, 60, 290, 0, 0, 3, 200, 7], [2 ** 31 - 1] * 4 + [-2 ** 31] * 5):
        out = [torch.full((T, H, d), 7.0, dtype=dtype, device=dev) for _ in range(2)]
        got = omnimem_read_kv_quant(cache, T, i32(starts, dev), first=None if first is None else i32(first, dev), out=out)
        assert got[0] is out[0] and got[1] is out[1]
        want = [torch.full((T, H, d), 7.0, dtype=torch.float64) for _ in range(2)]
        quant_oracle.read(k, v, scales, table, lens, T, starts, first, S, *want)
        for a, b in zip(out, want):
            a = a.double().cpu()
            assert torch.equal(torch.isnan(a), torch.isnan(b))
            # c * s rounded to fp32 (4 bits times 24), then to the type
            tol = (2.0 ** -24 + (2.0 ** -8 if dtype is BF16 else 0)) * b.abs().nan_to_num()
            assert ((a - b).abs().nan_to_num() <= tol).all()
    # one token for each
    short = SeqKVCacheQuant(cache.k_pages, cache.v_pages, cache.scales, cache.page_table, cache.seq_lens.clamp(max=64), S)
    a = omnimem_read_kv_quant(short, len(lens), dtype=dtype)
    want = [torch.zeros((len(lens), H, d), dtype=torch.float64) for _ in range(2)]
    quant_oracle.read(k, v, scales, table, short.seq_lens.tolist(), len(lens), None, None, S, *want)
    for x, w in zip(a, want):
        assert torch.equal(x.double().cpu().nan_to_num(-1), w.float().to(dtype).double().nan_to_num(-1))


def test_one_token_read_from_inside(dev):
    """One token a sequence at a place of its own, without starts; places that a sequence does not have are 0."""
    g = torch.Generator().manual_seed(17)
    lens = [5, 64, 130, 0, -2, 300, 64]
    first = [4, 0, 129, 0, 0, 300, -1]
    table, P = tables(lens, 64, 64, g)
    k, v, scales = pools(P, 2, 64, 64, g)
    cache = SeqKVCacheQuant(k.to(dev).view(F8), v.to(dev).view(F8), scales.to(dev), i32(table, dev), i32(lens, dev))
    want = [torch.zeros((7, 2, 64), dtype=torch.float64) for _ in range(2)]
    quant_oracle.read(k, v, scales, table, lens, 7, None, first, 64, *want)
    for dtype in (F32, BF16):
        got = omnimem_read_kv_quant(cache, 7, first=i32(first, dev), dtype=dtype)
        for x, w in zip(got, want):
            assert torch.equal(x.double().cpu().nan_to_num(-1), w.float().to(dtype).double().nan_to_num(-1))
            assert (x[3:] == 0).all()


def test_what_is_appended_is_read(dev):
    """Values that e4m3 holds come back as they were, in bf16 and fp32."""
    g = torch.Generator().manual_seed(13)
    finite = torch.tensor([c for c in range(256) if c & 127 != 127], dtype=torch.uint8)
    x = quant_oracle.values(finite[torch.randint(0, len(finite), (500, 4, 128), generator=g)]).float()
    x[:, :, 5] = 448                                             # every block's scale is 1
    n = [200, 1, 64, 235]
    starts = [0, 200, 201, 265, 500]
    table, P = tables(n, 150, 64, g)
    for dtype in (F32, BF16):
        k, v, scales = pools(P, 4, 64, 128, g)
        cache = SeqKVCacheQuant(k.to(dev).view(F8), v.to(dev).view(F8), scales.to(dev), i32(table, dev), i32(n, dev), 150)
        omnimem_append_kv_quant(cache, x.to(dtype).to(dev), -x.to(dtype).to(dev), i32(starts, dev))
        for to in (BF16, F32):
            a, b = omnimem_read_kv_quant(cache, 500, i32(starts, dev), dtype=to)
            assert torch.equal(a.float().cpu(), x) and torch.equal(b.float().cpu(), -x)
    assert omnimem_read_kv_quant(cache, 0, i32([0] * 5, dev))[0].shape == (0, 4, 128)


# ------------------------------------------------------------------------- copy

@pytest.mark.parametrize("H,B,d", [(1, 64, 64), (3, 64, 128), (300, 128, 64), (8, 128, 128)])
@pytest.mark.parametrize("layers", [None, 3])
def test_copies(dev, H, B, d, layers):
    say(f"copy H={H} B={B} d={d} layers={layers}")
    P = 9
    g = torch.Generator(device=dev).manual_seed(14)
    lead = () if layers is None else (layers + 1,)
    k, v = (torch.randint(0, 256, lead + (P, H, B, d), generator=g, device=dev, dtype=torch.uint8) for _ in range(2))
    scales = torch.randn(lead + (P + 2, H, 2), generator=g, device=dev)
    ks, vs, ss = (k[:layers], v[:layers], scales[:layers, :P]) if layers else (k, v, scales[:P])    # layers' scales lie apart
    pairs = [(0, 5), (1, 2), (0, 3), (-1, 4), (4, -7), (6, P), (P, 6), (2 ** 31 - 1, 8), (7, 8), (8, 1)]
    for count in (9, 2, 0, -3, 100):
        wk, wv, ws = ks.clone(), vs.clone(), ss.clone()
        n = min(max(count, 0), 9)
        for s, t in pairs[:n]:
            if 0 <= s < P and 0 <= t < P:
                for x, y in ((wk, ks), (wv, vs), (ws, ss)):
                    if layers:
                        x[:, t] = y[:, s].clone()
                    else:
                        x[t] = y[s].clone()
        rest = k[-1].clone(), scales[..., P:, :, :].clone()
        omnimem_copy_pages_quant(ks.view(F8), vs.view(F8), ss, i32(pairs[:9], dev), i32([count], dev))
        torch.cuda.synchronize()
        assert torch.equal(ks, wk) and torch.equal(vs, wv) and torch.equal(ss, ws)
        if layers:
            assert torch.equal(k[-1], rest[0])
        assert torch.equal(scales[..., P:, :, :], rest[1])


def test_copies_past_the_caches(dev):
    """More bytes than the memory-side cache holds, every page's scales with it."""
    g = torch.Generator(device=dev).manual_seed(15)
    P, H = 3000, 12
    k, v = (torch.randint(0, 256, (P, H, 64, 128), generator=g, device=dev, dtype=torch.uint8) for _ in range(2))
    scales = torch.randn((P, H, 2), generator=g, device=dev)
    ids = torch.randperm(P, generator=g, device=dev).int()
    pairs = torch.stack([ids[:1400], ids[1400:2800]], 1).contiguous()
    omnimem_copy_pages_quant(k.view(F8), v.view(F8), scales, pairs)
    s, t = pairs.long().unbind(1)
    assert torch.equal(k[t], k[s]) and torch.equal(v[t], v[s]) and torch.equal(scales[t], scales[s])


def test_random_appends(dev):
    rng = random.Random(16)
    for case in range(12):
        d, B, H = rng.choice([64, 128]), rng.choice([64, 128]), rng.randrange(1, 5)
        S = rng.choice([B, B, rng.randrange(1, 300)])
        lens = [rng.randrange(0, 500) for _ in range(rng.randrange(1, 9))]
        new = [rng.randrange(0, t + 3) for t in lens]
        dtype = rng.choice([BF16, F32])
        say(f"append case {case}: {dtype} d={d} B={B} H={H} S={S} lens={lens} new={new}")
        g = torch.Generator().manual_seed(case)
        table, P = tables(lens, S, B, g)
        k, v, scales = pools(P, H, B, d, g)
        nk, nv = (torch.randn((sum(new), H, d), generator=g).to(dtype) for _ in range(2))
        starts = [sum(new[:i]) for i in range(len(new) + 1)]
        append_and_compare(dev, k, v, scales, table, lens, nk, nv, starts, S, B)
