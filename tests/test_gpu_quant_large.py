"""Appends and reads of the 8-bit cache of a size that other kernels take: more (block, head) pairs than an append has
workgroups, and outputs that are stored past the caches (over 96 MB of codes, over 288 MB of rows)."""
import pytest
import torch

import quant_oracle
from parity import say
from paper_2605_30519_amd import SeqKVCacheQuant, omnimem_append_kv_quant, omnimem_read_kv_quant

pytestmark = pytest.mark.gpu
BF16, F32, F8, U8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.uint8


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    yield d
    torch.cuda.empty_cache()


def test_workgroups_with_two_units(dev):
    """5,600,000 (block, head) pairs, of which a workgroup has the w-th and the (w + 2^22)-th: sequences whose units are
    first and second ones of the same workgroups, begun blocks, not begun ones, infinities and NaN among them, and
    units without a page in front of units with one."""
    N, H, d, B = 140000, 40, 64, 64
    turn = 2 ** 22 // H                                           # 104,857 sequences and 24 heads
    g = torch.Generator(device=dev).manual_seed(1)
    lens = torch.ones(N, dtype=torch.int32, device=dev)
    some = [0, 7, 8, 500, 501, turn, 7 + turn, 8 + turn, 9 + turn, 500 + turn, 501 + turn, 502 + turn, 700 + turn, N - 2, N - 1]
    for i, n in zip(some, [1, 30, 1, 64, 2, 17, 1, 40, 1, 63, 1, 33, 50, 1, 9]):
        lens[i] = n
    P = len(some)
    table = torch.full((N, 1), -1, dtype=torch.int32, device=dev)
    table[torch.tensor(some, device=dev), 0] = torch.randperm(P, generator=g, device=dev).int()
    x = torch.randn((N, H, d), generator=g, device=dev).to(BF16)
    x[some[1::2]] *= 64
    x[some[2], :, 5] = float("inf")
    x[some[8], 3::2, 60] = float("nan")
    k, v = (torch.randint(0, 256, (P, H, B, d), generator=g, device=dev, dtype=U8) for _ in range(2))
    scales = torch.exp2(torch.randint(-12, 3, (P, H, 2), generator=g, device=dev).float())
    wk, wv, ws = k.cpu(), v.cpu(), scales.cpu()
    say(f"append {N} tokens to {H} heads")
    omnimem_append_kv_quant(SeqKVCacheQuant(k.view(F8), v.view(F8), scales, table, lens), x, x)
    torch.cuda.synchronize()
    assert N * H > 2 ** 22 and min(i for i in some if i * H >= 2 ** 22) < N
    new = x[some].cpu()
    quant_oracle.append(wk, wv, ws, table[some].tolist(), lens[some].tolist(), new, new, None, B)
    assert quant_oracle.same_codes(k, wk) and quant_oracle.same_codes(v, wv) and torch.equal(scales.cpu(), ws)


def history(dev, g, H, d, B, S, lens):
    """A pool of random codes and scales, and a table in which one block of the second sequence is not resident."""
    bpc = -(-S // B)
    nb = [t // S * bpc + -(-(t % S) // B) for t in lens]
    P = sum(nb)
    order = torch.randperm(P, generator=g, device=dev).int()
    table = torch.full((len(lens), max(nb)), -1, dtype=torch.int32, device=dev)
    at = 0
    for i, n in enumerate(nb):
        table[i, :n] = order[at:at + n]
        at += n
    table[1, nb[1] // 2] = -1
    k, v = (torch.randint(0, 127, (P, H, B, d), generator=g, device=dev, dtype=U8) for _ in range(2))
    scales = torch.exp2(torch.randint(-12, 1, (P, H, 2), generator=g, device=dev).float())
    return k, v, scales, table, torch.tensor(lens, dtype=torch.int32, device=dev)


def starts_of(new, dev):
    return torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device=dev)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,B,S", [(64, 64, 64), (128, 64, 1000), (64, 128, 128), (128, 128, 128)])
def test_large_appends(dev, dtype, d, B, S):
    """The codes and scales of appends sequence by sequence, which are stored through the caches."""
    H = 8
    g = torch.Generator(device=dev).manual_seed(2)
    each = 52_000_000 // (8 * H * d)                              # of 8 sequences
    new = [each + 37 * i for i in range(8)]
    lens = [n + t for n, t in zip(new, (0, 1, 63, 64, 65, 100, 130, 2000))]
    T = sum(new)
    assert 2 * T * H * d > 96 << 20 > 2 * 2 * max(new) * H * d
    say(f"append {T} tokens {dtype} d={d} B={B} S={S}")
    k, v, scales, table, lens = history(dev, g, H, d, B, S, lens)
    x = torch.randn((T, 2, H, d), generator=g, device=dev)
    x *= torch.exp(torch.randn((T, 1, H, 1), generator=g, device=dev))
    x[17, :, 3, 9], x[T // 2, :, 1, 1], x[T - 5, :, :, 0] = float("inf"), float("nan"), -float("inf")
    x = x.to(dtype)
    nk, nv = x[:, 0], x[:, 1]
    k1, v1, s1 = k.clone(), v.clone(), scales.clone()
    omnimem_append_kv_quant(SeqKVCacheQuant(k.view(F8), v.view(F8), scales, table, lens, S), nk, nv, starts_of(new, dev))
    at = 0
    for i, n in enumerate(new):
        one = SeqKVCacheQuant(k1.view(F8), v1.view(F8), s1, table[i:i + 1], lens[i:i + 1], S)
        omnimem_append_kv_quant(one, nk[at:at + n], nv[at:at + n], starts_of([n], dev))
        at += n
    torch.cuda.synchronize()
    assert torch.equal(scales, s1) and torch.equal(k, k1) and torch.equal(v, v1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,B,S", [(128, 64, 64), (64, 128, 1000)])
@pytest.mark.parametrize("inside", [False, True])
def test_large_reads(dev, dtype, d, B, S, inside):
    """The rows of reads sequence by sequence, which are stored through the caches; rows of no sequence stay."""
    H = 8
    g = torch.Generator(device=dev).manual_seed(3)
    each = 160_000_000 // dtype.itemsize // (8 * H * d)
    n = [each + 41 * i for i in range(8)]
    lens = [t + e for t, e in zip(n, (0, 1, -100, 64, 65, 100, 130, 2000))]
    T = sum(n) + 5
    assert 2 * T * H * d * dtype.itemsize > 288 << 20 > 2 * 2 * max(n) * H * d * dtype.itemsize
    say(f"read {T} tokens {dtype} d={d} B={B} S={S}")
    k, v, scales, table, lens = history(dev, g, H, d, B, S, lens)
    scales *= 1 + torch.rand(scales.shape, generator=g, device=dev)
    cache = SeqKVCacheQuant(k.view(F8), v.view(F8), scales, table, lens, S)
    first = torch.tensor([0, 1, 7, 64, 3, 0, 200, 1], dtype=torch.int32, device=dev) if inside else None
    out = [torch.full((T, H, d), 7.0, dtype=dtype, device=dev) for _ in range(2)]
    omnimem_read_kv_quant(cache, T, starts_of(n, dev), first=first, out=out)
    at = 0
    for i, m in enumerate(n):
        one = SeqKVCacheQuant(cache.k_pages, cache.v_pages, scales, table[i:i + 1], lens[i:i + 1], S)
        part = omnimem_read_kv_quant(one, m, starts_of([m], dev), first=None if first is None else first[i:i + 1], dtype=dtype)
        for a, b in zip(out, part):
            assert torch.equal(a[at:at + m], b)
        at += m
    assert all((a[at:] == 7).all() for a in out)
