"""omnimem_copy_pages and omnimem_copy_pages_quant around the number of pieces up to which each is a workgroup's of
its own (1,536 of 16 KB): lists as long as that, one pair longer, and long lists of which the device counts few."""
import pytest
import torch

from parity import say
from paper_2605_30519_amd import omnimem_copy_pages, omnimem_copy_pages_quant

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


# dtype, heads, block, dims, layers, pairs of 1,536 pieces
CASES = [(torch.bfloat16, 12, 64, 128, 1, 64), (torch.float32, 3, 64, 64, 4, 64), (torch.bfloat16, 1, 64, 64, 1, 768),
         (torch.uint8, 12, 64, 128, 2, 64), (torch.uint8, 1, 64, 64, 1, 768), (torch.uint8, 3, 128, 128, 4, 64)]


@pytest.mark.parametrize("dtype,H,B,d,layers,edge", CASES)
def test_one_piece_a_workgroup(dev, dtype, H, B, d, layers, edge):
    g = torch.Generator(device=dev).manual_seed(1)
    n = edge + 1
    P = 2 * n
    size = torch.empty(0, dtype=dtype).element_size()
    k0, v0 = (torch.randint(0, 256, (layers, P, H, B, d * size), generator=g, device=dev, dtype=torch.uint8).view(dtype)
              for _ in range(2))
    s0 = torch.randn((layers, P, H, 2), generator=g, device=dev)
    order = torch.randperm(P, generator=g, device=dev).int()
    pairs = torch.stack([order[:n], order[n:]], 1).contiguous()
    pairs[3, 0], pairs[7, 1] = -1, P                              # no such pages
    for most, count in ((edge - 1, None), (edge, None), (n, None), (n, edge), (n, edge - 1), (n, 1), (n, 0), (n, -5)):
        say(f"copy {dtype} H={H} layers={layers} list={most} count={count}")
        k, v, s = k0.clone(), v0.clone(), s0.clone()
        c = None if count is None else torch.tensor([count], dtype=torch.int32, device=dev)
        if dtype is torch.uint8:
            omnimem_copy_pages_quant(k.view(F8), v.view(F8), s, pairs[:most], c)
        else:
            omnimem_copy_pages(k, v, pairs[:most], c)
        take = pairs[:most if count is None else max(count, 0)].long()
        take = take[(take >= 0).all(1) & (take < P).all(1)]
        for got, was in ((k, k0), (v, v0), (s, s0)):
            want = was.clone()
            if got is not s or dtype is torch.uint8:
                want[:, take[:, 1]] = was[:, take[:, 0]]
            assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))
