"""omnimem_append_kv_quant's second rounding of a begun block, where the block's own scale is no power of two: the
products c * own / new lie beside the middle of two e4m3 numbers, closer to it than fp32 tells apart."""
import pytest
import torch

import quant_oracle
from paper_2605_30519_amd import SeqKVCacheQuant, omnimem_append_kv_quant

F8 = torch.float8_e4m3fn


def own_scales():
    """fp32 numbers s in [1, 2) beside t / c, c a code's significand and t a middle of two neighbours', and
    those next to them."""
    found = set()
    for c in range(8, 16):
        for t in range(17, 32, 2):
            s = torch.tensor(t / 2 / c, dtype=torch.float64)
            s = (s * 2 if s < 1 else s).float()
            for to in (0.0, 4.0):
                found |= {float(s), float(torch.nextafter(s, torch.tensor(to)))}
    return torch.tensor(sorted(s for s in found if 1 < s < 2))


def products(s):
    """All codes' values times own / new, exact (4 bits times 24), and those products rounded to fp32 first."""
    finite = quant_oracle.VALUES[[c for c in range(256) if c & 127 != 127]]
    exact = finite[None] * (s.double() / 2)[:, None]
    return exact, exact.float().double()


def test_the_scales_tell_two_roundings_from_one():
    exact, twice = products(own_scales())
    assert int((quant_oracle.codes(exact) != quant_oracle.codes(twice)).sum()) > 100


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,B", [(64, 64), (128, 128)])
def test_earlier_codes_are_rounded_once(dtype, d, B):
    dev = torch.device("cuda:0")
    s = own_scales()
    P = s.numel()
    n = 256 // d                                                 # tokens that hold every code
    k = torch.zeros((P, 1, B, d), dtype=torch.uint8)
    k[:, 0, :n] = torch.arange(256, dtype=torch.uint8).view(n, d)
    v = k.flip(3).contiguous()
    scales = torch.stack([s, s.flip(0)], 1).view(P, 1, 2).contiguous()
    table, lens = [[p] for p in range(P)], [n + 1] * P
    new = torch.zeros((P, 1, d), dtype=dtype)                    # needs no scale: the block's own, rounded up to 2
    gk, gv, gs = k.to(dev), v.to(dev), scales.to(dev)
    cache = SeqKVCacheQuant(gk.view(F8), gv.view(F8), gs, torch.tensor(table, dtype=torch.int32, device=dev),
                            torch.tensor(lens, dtype=torch.int32, device=dev))
    omnimem_append_kv_quant(cache, new.to(dev), new.to(dev))
    quant_oracle.append(k, v, scales, table, lens, new, new, None, B)
    assert torch.equal(gs.cpu(), scales) and (scales == 2).all()
    assert quant_oracle.same_codes(gk, k) and quant_oracle.same_codes(gv, v)
