"""Attention with masked and reshaped scores: row lists whose offsets descend are refused on the device, and leave nothing behind."""
import numpy as np
import pytest
import torch

from paper_2603_08026_amd import binding as Bd
from synth import workload as W
from tests import scored_shapes as S
from tests.test_gpu_pages import TD, dev, ints, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("s", S.SPLITS, ids=lambda s: "-".join(str(x) for x in s))
def test_offsets_that_descend(s):
    """Nothing is written, the status word says so, and later calls on the context, whose keys are split among workgroups that count each other, are as before."""
    say("offsets that descend", *s)
    g = W.philox(61, *s)
    ctx = Bd.Context(Bd.LayerCfg(256, s.H, s.Hkv, s.dh, 256, 1 if s.pages else s.B, s.room, 0, Bd.F32 if s.t == "f32" else Bd.BF16, 1e-5, 1e4))
    per = s.cap // s.B
    off = np.arange(s.B + 1) * per
    pos = np.concatenate([np.sort(g.choice(s.L, per, replace=False)) for _ in range(s.B)])
    q = dev(g.standard_normal((s.cap, s.H, s.dh)), s.t)
    scores = Bd.Scores(block=1)
    lengths = ints(s.L - 3 * np.arange(s.B)) if s.lengths else None
    if s.pages:
        P, n_pages = 16, 40
        pages = Bd.Pages(*(dev(g.standard_normal((n_pages, s.Hkv, P, s.dh)), s.t) for _ in range(2)), ints(g.integers(0, n_pages, (s.B, s.L // P))))
    else:
        k, v = (dev(g.standard_normal((s.B, s.L, s.Hkv, s.dh)), s.t) for _ in range(2))

    def call(offsets, out):
        if s.pages:
            ctx.paged_attention(q, pages, Bd.PageRows(ints(offsets), ints(pos), ints(pos)), lengths, out, scores)
        else:
            ctx.partial_attention_masked(q, k, v, Bd.IndexList(ints(pos + np.arange(s.B).repeat(per) * s.L), ints(offsets)), s.B, s.L, out, scores, lengths)
        return ctx.poll_status()

    empty = lambda: torch.full((s.cap, s.H * s.dh), 7.0, dtype=TD[s.t], device="cuda")  # noqa: E731
    want = empty()
    assert call(off, want) == 0 and torch.all(torch.isfinite(want)) and not torch.any((want == 7.0).all(-1))
    twice, back, short = off.copy(), off.copy(), off.copy()
    twice[1], twice[2] = s.cap, 0       # rows named twice and more
    back[-2] = s.cap + 5                # the last sequence ends before it starts
    short[1], short[2] = per + 1, per   # by one row
    for bad in (twice, back, short):
        out = empty()
        assert call(bad, out) == Bd.ERR_INVALID_ARG
        assert torch.all(out == 7.0)
        for _ in range(2):
            out = empty()
            assert call(off, out) == 0 and torch.equal(out, want)
    ahead = off.copy()                  # rows ahead of the first sequence stay
    ahead[0] = 1
    out = empty()
    assert call(ahead, out) == 0
    assert torch.all(out[0] == 7.0) and not torch.any((out[1:] == 7.0).all(-1))
    ctx.close()
