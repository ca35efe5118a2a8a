"""The plain models of the 8-bit cache against things other than themselves (CPU): e4m3's known
numbers, torch's own e4m3 conversion, scales by hand."""
import torch

import quant_oracle as qo

F8 = torch.float8_e4m3fn


def test_values_are_torchs():
    c = torch.arange(256, dtype=torch.uint8)
    want = c.view(F8).double()
    got = qo.values(c)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.isnan(got).sum() == 2
    assert torch.equal(got.nan_to_num(0.5), want.nan_to_num(0.5))
    assert got[0x7e] == 448 and got[0x08] == 2.0 ** -6 and got[0x01] == 2.0 ** -9 and got[0xb8] == -1


def test_rounding_is_torchs():
    x = qo.VALUES[:127]
    mid = (x[1:] + x[:-1]) / 2
    x = torch.cat([x, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20), torch.randn(4000, dtype=torch.float64) * 30])
    x = torch.cat([x, -x]).clamp(-448, 448)
    assert torch.equal(qo.codes(x), x.float().to(F8).view(torch.uint8))
    assert qo.codes(torch.tensor([float("inf"), -float("inf"), float("nan")])).tolist() == [127] * 3


def test_scales_by_hand():
    for most, e in ((448.0, 0), (448.25, 1), (449.0, 1), (224.0, -1), (1.75, -8), (1.76, -7), (0.0, -110), (2.0 ** -101, -109),
                    (1.75 * 2.0 ** -102, -110), (3.4e38, 120)):
        assert qo.needed(torch.tensor([-most, 0.0, float("nan"), float("inf")], dtype=torch.float64)) == e, most


def test_append_by_hand():
    """One head of four dims; blocks of four tokens: a second append raises the scale of a begun block."""
    k = torch.full((2, 1, 4, 4), 0x55, dtype=torch.uint8)
    v, scales = k.clone(), torch.full((2, 1, 2), float("nan"))
    new = torch.tensor([[448.0, -16, 1, 2.0 ** -9]])[:, None]
    qo.append(k, v, scales, [[1, -1]], [1], new, new * 2, [0, 1], 4)
    assert scales[1].tolist() == [[1.0, 2.0]] and torch.isnan(scales[0]).all()
    assert k[1, 0, 0].tolist() == v[1, 0, 0].tolist() == [0x7e, 0xd8, 0x38, 0x01] and (k[1, 0, 1:] == 0x55).all()
    qo.append(k, v, scales, [[1, -1]], [2], new * 4, new, [0, 1], 4)
    assert scales[1].tolist() == [[4.0, 2.0]]
    assert k[1, 0, 0].tolist() == [0x6e, 0xc8, 0x28, 0x00]       # a quarter: exponents by two, 2^-11 rounds to 0
    assert k[1, 0, 1].tolist() == [0x7e, 0xd8, 0x38, 0x01]
    assert v[1, 0, 1].tolist() == [0x76, 0xd0, 0x30, 0x00]       # half of 2^-9: a tie, to the even 0
    assert (k[0] == 0x55).all() and (k[1, 0, 2:] == 0x55).all()
