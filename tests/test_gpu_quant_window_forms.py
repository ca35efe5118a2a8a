"""omnimem_decode_attn_quant for more than 16 query heads a key head under windows, over tables far longer than them: the
form is chosen by what the window leaves."""
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
