"""omnimem_seq_update where a batch drains: no new rows, or one empty one, over tables and pools of
every size, with scratch of exactly the size asked for, full of another use's bits."""
import pytest
import torch

import seq_oracle
from parity import say
from paper_2605_30519_amd import omnimem_seq_update, omnimem_seq_workspace_bytes

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


@pytest.mark.parametrize("N,M,P", [(3, 10, 30), (256, 65, 4000), (2000, 2, 100), (3, 10, 17000), (40, 30, 1 << 20), (0, 5, 20000),
                                   (5000, 9, 0)])
@pytest.mark.parametrize("fill", [255, 0, 85])
def test_rows_end(dev, N, M, P, fill):
    say(f"drain N={N} M={M} P={P} fill={fill}")
    table = (torch.arange(N * M, dtype=torch.int32).view(N, M) * 7 % max(P, 1)).to(dev)
    lens = (torch.arange(N, dtype=torch.int32) * 37 % (64 * M + 1)).to(dev)
    empty = torch.empty(0, dtype=torch.int32, device=dev)
    # every sequence ends
    need = omnimem_seq_workspace_bytes(table, lens, P, 64, 0)
    around = torch.full((need + (1 << 20),), fill, dtype=torch.uint8, device=dev)
    u = omnimem_seq_update(table, lens, P, 64, empty, empty, empty, workspace=around[:need])
    assert u.info.tolist() == [0, 0, 0, 0]
    assert u.page_table.shape == (0, M) and u.seq_lens.shape == (0,) and u.copies.shape == (0, 2)
    assert (around[need:] == fill).all()
    # and one takes their place, without a token or with as many as two pages hold, or one row goes on
    for parent, grow in ([-1], [0]), ([-1], [min(100, 64 * M)]), ([min(N, 2)], [0]):
        need = omnimem_seq_workspace_bytes(table, lens, P, 64, 1)
        around = torch.full((need + (1 << 20),), fill, dtype=torch.uint8, device=dev)
        u = omnimem_seq_update(table, lens, P, 64, torch.tensor(parent, dtype=torch.int32, device=dev), None,
                               torch.tensor(grow, dtype=torch.int32, device=dev), workspace=around[:need])
        rows, want, copies, info = seq_oracle.update(table.tolist() or [[-1] * M], lens.tolist() or [0], P, 64, 64,
                                                     parent if N else [-1], None, grow)
        assert u.info.tolist() == info and u.page_table.tolist() == rows and u.seq_lens.tolist() == want
        assert u.copies.tolist() == [list(c) for c in copies] + [[-1, -1]] * (1 - len(copies))
        assert (around[need:] == fill).all()
