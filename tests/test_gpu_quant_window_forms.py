"""omnimem_decode_attn_quant for more than 16 query heads a key head: its forms are chosen by what a window leaves of a table
and by the queries' type."""
import pytest
import torch

from parity import say
from test_gpu_quant_decode import BF16, F32, build, check, dev, queries  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 128), (BF16, 64), (F32, 64)])
@pytest.mark.parametrize("G", [17, 24, 40])
def test_windows_over_long_tables(dev, dtype, d, G):  # noqa: F811
    lens = [200, 0, 70, 3000]
    cache, g = build(dev, 2, d, 64, 64, lens, 13, extra_blocks=9000)
    q = queries(dev, dtype, 4, 2 * G, d, g)
    # a workgroup's items, pairs of waves over a line, both column tiles in a wave
    for window in (600, 2700, 400000):
        say(f"decode windows {dtype} d={d} G={G} window={window}")
        check(cache, q, window)
    assert all(torch.equal(a, b) for a, b in zip(check(cache, q, 2 ** 31 - 1), check(cache, q)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_more_items_than_cus(dev, dtype, d):  # noqa: F811
    """264 items over 346 MB of capacity (heads of 128): both column tiles in a wave for bf16, pairs for fp32."""
    lens = [13 * i for i in range(33)]
    say(f"decode items {dtype} d={d}")
    cache, g = build(dev, 8, d, 64, 64, lens, 14, extra_blocks=73)
    check(cache, queries(dev, dtype, 33, 8 * 24, d, g))
