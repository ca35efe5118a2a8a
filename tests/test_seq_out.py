"""The binding's buffers of a table call, on the CPU: a compaction's lengths are the given ones."""
import pytest
import torch

from paper_2605_30519_amd import omnimem as om

I32 = torch.int32


def test_a_compaction_keeps_the_given_lengths():
    lens = torch.tensor([5, 9], dtype=I32)
    for held in (torch.full((2,), 77, dtype=I32), None):
        out = om.SeqUpdate(torch.zeros((2, 3), dtype=I32), held, torch.zeros((4, 2), dtype=I32), torch.zeros(4, dtype=I32))
        made = om._seq_out(out, 2, 3, 4, lens, "cpu")
        assert made.seq_lens is lens
        assert made.page_table is out.page_table and made.copies is out.copies and made.info is out.info
    made = om._seq_out(None, 2, 3, 4, lens, "cpu")
    assert made.seq_lens is lens and made.copies.shape == (4, 2)


def test_an_update_needs_lengths_of_its_own():
    out = om.SeqUpdate(torch.zeros((2, 3), dtype=I32), None, torch.zeros((2, 2), dtype=I32), torch.zeros(4, dtype=I32))
    with pytest.raises(ValueError, match="out.seq_lens must be a tensor"):
        om._seq_out(out, 2, 3, 2, None, "cpu")
    out.seq_lens = torch.zeros(2, dtype=I32)
    assert om._seq_out(out, 2, 3, 2, None, "cpu") is out
