"""omnimem_seq_compact into the caller's buffers: the result carries the lengths that were given, whatever
lies in the buffers, so that the cache under its tables attends to the same tokens."""
import pytest
import torch

import test_gpu_seq_decode as base
from paper_2605_30519_amd import SeqUpdate, omnimem_append_kv, omnimem_copy_pages, omnimem_decode_attn, omnimem_seq_compact

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


def buffers(cache, lens):
    i32 = dict(dtype=torch.int32, device=cache.page_table.device)
    return SeqUpdate(torch.full(cache.page_table.shape, 77, **i32), lens,
                     torch.full((cache.k_pages.shape[0] // 2, 2), 77, **i32), torch.full((4,), 77, **i32))


def compacted(cache, out):
    B = cache.k_pages.shape[2]
    u = omnimem_seq_compact(cache.page_table, cache.seq_lens, cache.k_pages.shape[0], B, out=out)
    omnimem_copy_pages(cache.k_pages, cache.v_pages, u.copies, u.info)
    return u


@pytest.mark.parametrize("spare", [5, 20000])                     # one workgroup's table, and a larger pool
@pytest.mark.parametrize("junk", [0, 1, 64, 2 ** 31 - 1, None])
def test_lengths_stay(dev, spare, junk):
    cache, g = base.build(dev, torch.bfloat16, 1, 64, 64, 64, [300, 5, 0, 129], 40, spare=spare)
    cache.k_pages.nan_to_num_(0.0)
    cache.v_pages.nan_to_num_(0.0)
    q = base.queries(dev, torch.bfloat16, 4, 2, 64, g)
    want = omnimem_decode_attn(cache, q)
    lens = cache.seq_lens.clone()
    out = buffers(cache, None if junk is None else torch.full_like(lens, junk))
    u = compacted(cache, out)
    assert u.seq_lens is cache.seq_lens and torch.equal(u.seq_lens, lens)
    assert u.page_table is out.page_table and u.copies is out.copies and u.info is out.info
    assert junk is None or (out.seq_lens == junk).all()
    now = cache.after(u)
    got = omnimem_decode_attn(now, q)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # the next token goes behind the last one
    new = torch.full((2, 1, 64), 3.0, dtype=torch.bfloat16, device=dev)
    now.seq_lens = lens + torch.tensor([1, 1, 0, 0], dtype=torch.int32, device=dev)
    omnimem_append_kv(now, new, new, torch.tensor([0, 1, 2, 2, 2], dtype=torch.int32, device=dev))
    assert (now.k_pages[now.page_table[0, 4].long(), 0, 300 - 256] == 3).all()
    assert (now.k_pages[now.page_table[1, 0].long(), 0, 5] == 3).all()


def test_lengths_stay_in_a_graph(dev):
    """Captured with buffers of the caller's, as a step with fixed addresses needs them, and replayed."""
    cache, g = base.build(dev, torch.float32, 2, 64, 64, 64, [300, 70, 129], 41, spare=9)
    cache.k_pages.nan_to_num_(0.0)
    cache.v_pages.nan_to_num_(0.0)
    q = base.queries(dev, torch.float32, 3, 4, 64, g)
    first = cache.k_pages.clone(), cache.v_pages.clone()
    out = buffers(cache, torch.zeros_like(cache.seq_lens))
    o, lse = torch.empty_like(q), torch.empty((4, 3), device=dev)

    def step():
        u = compacted(cache, out)
        omnimem_decode_attn(cache.after(u), q, out=o, lse=lse)

    side = torch.cuda.Stream(device=dev)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([300, 70, 129], [299, 1, 0], [0, 70, 128]):
        cache.k_pages.copy_(first[0])
        cache.v_pages.copy_(first[1])
        cache.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        want = omnimem_decode_attn(cache, q)
        o.fill_(-9)
        out.seq_lens.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
