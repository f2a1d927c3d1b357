"""The binding of the drafting calls without a GPU: lists and tensors that the calls would read past their end, or as other numbers."""
from paper_2601_07667_amd import asl as libasl
from test_draft import recorded  # noqa: F401  (a fixture)


def test_an_empty_list_of_slots_is_a_list(recorded):
    """What the call is given for one is not what it is given for none, though a tensor without elements has no address."""
    import torch
    pages, i = libasl.make_pages(4, 2, 8, 16, 1, 1, 1), torch.zeros(4, dtype=torch.int32)
    path = torch.zeros(2, 4, dtype=torch.int32)
    accept = lambda slot: recorded.asl_pages_accept(pages, i, i, 1, i, i, path, i, 2, i, i, i, slot=slot)
    some = torch.zeros(5, dtype=torch.int64)
    for slot in (None, some[:0], some):
        accept(slot)
    none, empty, full = [seen[11:13] for seen in recorded.lib.seen]
    assert none == (None, 0) and full == (some.data_ptr(), 5)
    assert empty[0] and empty[1] == 0
