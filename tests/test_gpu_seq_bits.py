"""omnimem_decode_attn, bf16: the probabilities' bits.  Two keys carry nearly all of the weight and
their values cancel, so that an output of few bits shows how many the probabilities kept."""
import math

import pytest
import torch

from parity import say
from paper_2605_30519_amd import SeqKVCache, omnimem_decode_attn

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
B = 64


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


def cancelling(dev, N, H, G, d, t, seed):
    """N sequences of t tokens; each key head's keys at an even token and the next score about 9 and
    the others about 0, and those two tokens' values weigh each other out."""
    g = torch.Generator().manual_seed(seed)
    M = -(-t // B)
    q = (torch.randint(0, 2, (N, H, d), generator=g) * 2.0 - 1.0)
    k = 0.3 * torch.randn((N, M * B, H, d), generator=g)
    v = 0.1 * torch.randn((N, M * B, H, d), generator=g)
    at = 2 * torch.randint(0, t // 2, (N, H), generator=g)
    i, h = torch.arange(N)[:, None], torch.arange(H)[None]
    size = torch.rand((2, N, H, 1), generator=g) * 0.5 + 8.75
    k[i, at, h], k[i, at + 1, h] = q * size[0] / math.sqrt(d), q * size[1] / math.sqrt(d)
    k = k.to(BF16)
    score = lambda x: (q.double() * x.double()).sum(-1, keepdim=True) / math.sqrt(d)
    weight = torch.exp(score(k[i, at, h]) - score(k[i, at + 1, h]))
    first = torch.randn((N, H, d), generator=g).to(BF16)
    v[i, at, h], v[i, at + 1, h] = first.float(), (-weight * first.double()).float()
    v = v.to(BF16)
    pages = lambda x: x.view(N, M, B, H, d).transpose(2, 3).reshape(N * M, H, B, d).contiguous().to(dev)
    cache = SeqKVCache(pages(k), pages(v), torch.arange(N * M, dtype=torch.int32, device=dev).view(N, M),
                       torch.full((N,), t, dtype=torch.int32, device=dev))
    return cache, q.to(BF16).repeat_interleave(G, 1).to(dev), k[:, :t].double(), v[:, :t].double(), q.double()


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("N,H,G,t", [(4, 8, 4, 1500), (4, 2, 20, 1500), (8, 8, 4, 300), (8, 2, 20, 300), (128, 8, 1, 100),
                                     (32, 32, 17, 64)])
def test_probabilities_keep_more_than_bf16(dev, d, N, H, G, t):
    """Off by the scores' fp32 sums and the sums over t keys as in seq_oracle.decode, by 3 * 2^-16 of
    each weight for its two bf16 pieces, and by the output's rounding, 2^-8 of itself."""
    say(f"decode bits d={d} N={N} H={H} G={G} t={t}")
    cache, q, k, v, q64 = cancelling(dev, N, H, G, d, t, d + t)
    out, _ = omnimem_decode_attn(cache, q)
    s = (k * q64[:, None]).sum(-1) / math.sqrt(d)
    mag = (k.abs() * q64[:, None].abs()).sum(-1).amax(1) / math.sqrt(d)
    w = torch.softmax(s, 1)[..., None]
    O, spread = (w * v).sum(1), (w * v.abs()).sum(1)
    u = 2.0 ** -24
    e = u * ((d + 3) * mag + 4 * s.abs().amax(1)) + 2.0 ** -22 + (t + 80) * u
    bound = spread * (2 * e[..., None] + 3 * 2.0 ** -16) + O.abs() * 2.0 ** -8
    off = (out.double().cpu().view(N, H, G, d) - O[:, :, None]).abs()
    assert (off - bound[:, :, None]).max() <= 0, f"{(off / bound[:, :, None]).max():.3g} times the bound"


@pytest.mark.parametrize("N,H,G,t", [(2, 2, 4, 2000), (3, 2, 20, 200), (128, 8, 1, 100)])
def test_infinite_values_stay_infinite(dev, N, H, G, t):
    """A token's infinite value gives an infinite output, of its sign, and leaves the other dims alone."""
    cache, q, _, _, _ = cancelling(dev, N, H, G, 128, t, 3)
    plain, _ = omnimem_decode_attn(cache, q)
    for tok in (0, 37, t - 1):
        page = cache.page_table[:, tok // B].long()
        v = cache.v_pages.clone()
        v[page, :, tok % B, 5] = math.inf
        v[page, :, tok % B, 77] = -math.inf
        out, _ = omnimem_decode_attn(SeqKVCache(cache.k_pages, v, cache.page_table, cache.seq_lens), q)
        assert (out[..., 5] == math.inf).all() and (out[..., 77] == -math.inf).all()
        rest = [x for x in range(128) if x not in (5, 77)]
        assert torch.equal(out[..., rest], plain[..., rest])
