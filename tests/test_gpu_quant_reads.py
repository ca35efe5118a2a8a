"""omnimem_read_kv_quant of many rows a sequence, bit by bit: a code times its scale rounded to fp32, and that to the
type (the product of a code and an fp32 number is exact in fp64)."""
import pytest
import torch

import quant_oracle
from parity import say
from paper_2605_30519_amd import SeqKVCacheQuant, omnimem_read_kv_quant
from test_gpu_quant_pages import BF16, F32, F8, dev, i32, pools, tables  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,B,H,S", [(128, 64, 3, 64), (64, 64, 1, 100), (128, 128, 2, 300), (64, 128, 5, 128)])
def test_rows_have_the_bits_of_their_formula(dev, dtype, d, B, H, S):  # noqa: F811
    say(f"read bits {dtype} d={d} B={B} H={H} S={S}")
    g = torch.Generator().manual_seed(18)
    lens = [1, 64, 65, 300, 0, -3, 200, 2 ** 31 - 1, 150]
    table, P = tables([1, 64, 65, 300, 0, 0, 200, 250, 150], S, B, g, extra_blocks=0)
    table[6][1], table[8][0] = -1, P
    k, v, scales = pools(P, H, B, d, g)
    scales *= 1 + torch.rand(scales.shape, generator=g)
    n = [1, 70, 3, 300, 2, 5, 200, 9, 140]
    T = sum(n) + 4
    starts = [sum(n[:i]) for i in range(len(n) + 1)]
    cache = SeqKVCacheQuant(k.to(dev).view(F8), v.to(dev).view(F8), scales.to(dev), i32(table, dev), i32(lens, dev), S)
    for first in (None, [0, -2, 60, 290, 0, 0, 3, 200, 7], [0, 13, 0, 1, 0, -1, 100, 2, 149]):
        out = [torch.full((T, H, d), 7.0, dtype=dtype, device=dev) for _ in range(2)]
        omnimem_read_kv_quant(cache, T, i32(starts, dev), first=None if first is None else i32(first, dev), out=out)
        want = [torch.full((T, H, d), 7.0, dtype=torch.float64) for _ in range(2)]
        quant_oracle.read(k, v, scales, table, lens, T, starts, first, S, *want)
        for a, b in zip(out, want):
            assert torch.equal(a.double().cpu().nan_to_num(-1), b.float().to(dtype).double().nan_to_num(-1))
