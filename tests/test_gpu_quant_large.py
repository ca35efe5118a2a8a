"""Appends to the 8-bit cache of more (block, head) pairs than an append has workgroups."""
import pytest
import torch

import quant_oracle
from parity import say
from paper_2605_30519_amd import SeqKVCacheQuant, omnimem_append_kv_quant

pytestmark = pytest.mark.gpu
BF16, F8, U8 = torch.bfloat16, torch.float8_e4m3fn, torch.uint8


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
