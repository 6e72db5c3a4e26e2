"""Attention with masked and reshaped scores where scores are -infinity: such keys weigh nothing, and a row of nothing else is zero."""
import numpy as np
import pytest
import torch

from paper_2603_08026_amd import binding as Bd
from synth import workload as W
from tests import scored_shapes as S
from tests.test_gpu_masked_attention import run
from tests.test_gpu_pages import attend, dev, host, say, within
from tests.test_gpu_scored_kernels import context, name, parametrized

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which", ["all", "two thirds", "from the middle"])
@pytest.mark.parametrize("block", [0, 1])
@parametrized(S.INFINITE)
def test_scores_of_minus_infinity(s, block, which):
    say("scores of -infinity", name(s), block, which)
    g = W.philox(97, s.t, s.dh, s.cap)
    ctx = context(s)
    k, v = (dev(g.standard_normal((1, s.L, s.Hkv, s.dh)), s.t) for _ in range(2))
    idx = np.sort(g.choice(s.L, s.cap, replace=False))
    q = dev(g.standard_normal((s.cap, s.H, s.dh)), s.t)
    q[..., 0] = 0.5
    j = np.arange(s.L)
    out_of = {"all": j >= 0, "two thirds": j % 3 != 1, "from the middle": j >= s.L // 2}[which]
    at = torch.from_numpy(np.flatnonzero(out_of)).cuda()
    finite = host(k)[0]
    k[0, at, :, 0] = -float("inf")
    out = run(ctx, s.t, q, k, v, idx, np.array([0, s.cap]), 1, s.L, Bd.Scores(block=block))
    # the plain form with these keys out of sight: every row and the others in one document, the hidden ones in another
    want, tol = np.zeros((s.cap, s.H * s.dh)), np.zeros((s.cap, s.H * s.dh)) + 1e-30
    for n in range(s.cap):
        left = ~out_of & ((j <= idx[n]) if block else True)
        if left.any():
            want[n:n + 1], tol[n:n + 1] = attend(host(q)[n:n + 1], finite[left], host(v)[0, left], [0], s.t)
    within(out, want, tol, "rows")
    ctx.close()
