"""Row lists that the calls of normalised heads and of the 8-bit cache take.  No GPU needed: the list is looked at before anything else."""
import pytest
import torch

from paper_2603_08026_amd import binding as B


def _rows(idx, offsets, n_seq=2):
    return B.Context._rows(None, B.IndexList(idx, offsets), n_seq, 16, -1)


def test_a_list():
    c, n = _rows(torch.arange(6, dtype=torch.int32), torch.tensor([0, 3, 6], dtype=torch.int32))
    assert n == 6 and c._obj.cap == 6
    assert _rows(torch.zeros(0, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))[1] == 0


@pytest.mark.parametrize("idx,offsets", [
    (torch.arange(12, dtype=torch.int32)[::2], torch.tensor([0, 3, 6], dtype=torch.int32)),
    (torch.arange(6, dtype=torch.int32), torch.tensor([0, 9, 3, 9, 6], dtype=torch.int32)[::2]),
    (torch.zeros(1, dtype=torch.int32).expand(6), torch.tensor([0, 3, 6], dtype=torch.int32)),
    (torch.arange(6, dtype=torch.int32), torch.zeros(1, dtype=torch.int32).expand(3)),
])
def test_entries_that_do_not_lie_side_by_side(idx, offsets):
    with pytest.raises(ValueError, match="contiguous"):
        _rows(idx, offsets)


@pytest.mark.parametrize("idx,offsets", [
    (torch.arange(6), torch.tensor([0, 3, 6], dtype=torch.int32)),
    (torch.arange(6, dtype=torch.int32), torch.tensor([0, 3, 6])),
    (torch.arange(6, dtype=torch.int32), torch.tensor([0, 6], dtype=torch.int32)),
])
def test_other_types_and_too_few_offsets(idx, offsets):
    with pytest.raises(ValueError):
        _rows(idx, offsets)
