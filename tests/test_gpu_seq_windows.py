"""omnimem_decode_attn with windows past every row, over chunks of a token and more: every token counts,
as without a window."""
import pytest
import torch

import test_gpu_seq_decode as base
from parity import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("S,lens", [(1, [400, 129, 1, 0]), (2, [900, 300]), (100, [3000, 1])])
def test_a_window_past_every_row(dev, dtype, d, S, lens):
    say(f"decode whole windows {dtype} d={d} S={S}")
    cache, g = base.build(dev, dtype, 2, d, 64, S, lens, 30)
    q = base.queries(dev, dtype, len(lens), 6, d, g)
    want = base.check(cache, q)
    for window in (2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 3, max(lens)):
        got = base.check(cache, q, window)
        if window > 2 ** 30:                                     # split in the same way
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_many_rows_and_a_window_past_them(dev):
    """Over a thousand (sequence, head) items."""
    lens = [300 - i for i in range(130)]
    cache, g = base.build(dev, torch.bfloat16, 8, 64, 64, 1, lens, 31)
    q = base.queries(dev, torch.bfloat16, len(lens), 8, 64, g)
    some = [0, 1, 64, 129]
    out, lse = base.omnimem_decode_attn(cache, q, window=2 ** 31 - 1)
    O, L, ob, lb = base.seq_oracle.decode(q[some], cache.k_pages, cache.v_pages, cache.page_table[some],
                                          cache.seq_lens[some], 64, 1, 0, 0.125)
    assert ((out[some].double().cpu() - O).abs() <= ob).all() and ((lse[:, some].double().cpu() - L).abs() <= lb).all()
