"""Pages, rows and scores as the binding holds them: addresses are taken once, so the tensors that they name stay."""
import pytest
import torch

from paper_2603_08026_amd import binding as Bd


def holders():
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    k = torch.zeros(4, 2, 16, 64)
    return [(Bd.Pages(k, k.clone(), i32(2, 3)), ("k", "v", "table", "shape", "c"), ("k", "v", "table")),
            (Bd.PageRows(i32(3), i32(8), i32(8)), ("offsets", "pos", "slot", "cap", "c"), ("offsets", "pos", "slot")),
            (Bd.Scores(cap=2.0, block=1, prefix=i32(2), slopes=torch.zeros(4), doc=i32(2, 8)), ("cap", "block", "prefix", "slopes", "doc", "c"),
             ("prefix", "slopes", "doc"))]


@pytest.mark.parametrize("n", range(3))
def test_what_they_hold_cannot_be_exchanged(n):
    """An attribute that is set afterwards would change nothing in calls, or free a tensor whose address they still have."""
    h, names, tensors = holders()[n]
    for name in names:
        before = getattr(h, name)
        with pytest.raises(AttributeError):
            setattr(h, name, before)
        with pytest.raises(AttributeError):
            delattr(h, name)
        assert getattr(h, name) is before
    for name in tensors:
        assert getattr(h.c, name) == getattr(h, name).data_ptr()


def test_scores_hold_what_they_were_made_of():
    s = Bd.Scores(cap=2.0, block=3)
    assert (s.c.cap, s.c.block, s.c.prefix, s.c.slopes, s.c.doc) == (2.0, 3, None, None, None)
