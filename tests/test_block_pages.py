"""The block example's page table: every token of every sequence has a row of its own."""
import torch

from paper_2608_09160_amd.block import Pages


def test_slots_are_distinct_and_inside_the_pool():
    for sequences, tokens, page in ((1, 1, 16), (3, 70, 16), (4, 64, 32), (2, 33, 128)):
        pages = Pages(sequences, tokens, page, "cpu")
        seq = torch.arange(sequences).repeat_interleave(tokens)
        pos = torch.arange(tokens).repeat(sequences)
        slots = pages.slots(seq, pos)
        assert len(set(slots.tolist())) == sequences * tokens
        assert 0 <= slots.min() and slots.max() < pages.count * page
        # as the attention looks them up
        assert torch.equal(pages.table[seq, pos // page].long(), slots // page)
