"""Capped scores in fp32: as exact as the scores, whatever the cap and whichever kernel takes the rows."""
import math

import numpy as np
import pytest
import torch

from paper_2603_08026_amd import binding as Bd
from synth import workload as W
from tests import scored_shapes as S
from tests.test_gpu_pages import dev, host, ints, say, within

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("cap", [2.0 ** -20, 0.5, 30.0, 4096.0])
@pytest.mark.parametrize("s", S.CAPS, ids=lambda s: "-".join(str(x) for x in (s.H, s.Hkv, s.dh, s.cap, s.bq)))
def test_caps(s, cap):
    say("capped scores", *s, cap)
    g = W.philox(81, s.H, s.dh, s.cap)
    ctx = Bd.Context(Bd.LayerCfg(256, s.H, s.Hkv, s.dh, 256, 1, s.L, 0, Bd.F32, 1e-5, 1e4))
    k, v = (dev(g.standard_normal((1, s.L, s.Hkv, s.dh))) for _ in range(2))
    q = dev(0.1 * g.standard_normal((s.cap, s.H, s.dh)))
    idx = np.sort(g.choice(s.L, s.cap, replace=False))
    out = torch.zeros(s.cap, s.H * s.dh, device="cuda")
    ctx.partial_attention_masked(q, k, v, Bd.IndexList(ints(idx), ints([0, s.cap])), 1, s.L, out, Bd.Scores(cap=cap, block=1))
    torch.cuda.synchronize()
    qq, kk, vv = host(q), host(k)[0], host(v)[0]
    want, tol = np.zeros((s.cap, s.H, s.dh)), np.zeros((s.cap, s.H, s.dh)) + 1e-30
    seen = np.arange(s.L)[None] <= idx[:, None]
    for h in range(s.H):
        kb, vb = kk[:, h * s.Hkv // s.H], vv[:, h * s.Hkv // s.H]
        x = cap * np.tanh(qq[:, h] @ kb.T / math.sqrt(s.dh) / cap)
        # A score is off by its sum's roundings (dh products and sums, the scale), never more for being capped, and by a few of its own size: the
        # quotient by the cap (3), tanh (two steps of its last place: 4), cap in log2 units and the product (3), the difference to the maximum (2 of
        # the larger's size).  A weight by twice that, the exponential (2^-20) and the sum; a result by its own rounding.
        ds = (np.abs(qq[:, h]) @ np.abs(kb).T / math.sqrt(s.dh)).max(-1, keepdims=True) * (s.dh + 8) * U + 16 * U * np.abs(x).max(-1, keepdims=True)
        p = np.exp(np.where(seen, x, -np.inf))
        p /= p.sum(-1, keepdims=True)
        want[:, h] = p @ vb
        tol[:, h] += (np.expm1(2 * ds) + 2.0 ** -20 + s.L * U) * (p @ np.abs(vb)) * 1.05 + U * np.abs(want[:, h])
    within(out, want.reshape(s.cap, -1), tol.reshape(s.cap, -1), "rows")
    ctx.close()
