"""Layer steps over the cache in 8 bits of contexts that are no numbers: they reach the layer's output, and leave it again."""
import numpy as np
import pytest
import torch

from paper_2603_08026_amd.layer import Layer
from synth import workload as W
from tests.test_gpu_quant_cache import _dev, _layer, _lists

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("t,H,Hkv,dh", [("bf16", 4, 2, 128), ("bf16", 4, 4, 64), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_rows_that_are_no_numbers_are_salient(t, H, Hkv, dh, codes, bad):
    """One token of an input is no number: its sequence's contexts are none, so the dense step lists and writes every row, as do the step after
    it and, the input mended, the next dense one, which leaves what a layer that never met the token has.  A sparse step lists them too."""
    B, L = 2, 40
    print("[case] no numbers", t, H, Hkv, dh, codes, bad, flush=True)
    s, w = _layer(t, H, Hkv, dh, B, L, 131, True)
    lay, well = (Layer.from_shape(s, B, L, codes=codes) for _ in range(2))
    for z in (lay, well):
        z.set_weights(w)
    g = W.philox(132, t, dh)
    x0, x1 = (_dev(g.standard_normal((B * L, s.hidden)), t) for _ in range(2))
    broken = x0.clone()
    broken[3, 5] = bad
    dense = _lists(1, B, L, (L, L))[2]
    every = np.arange(B * L)

    def step(layer, x, il, tau):
        return layer.read_list(layer.layer_step_quant(x, il, tau))[0]

    for z in (lay, well):
        assert np.array_equal(step(z, x0, dense, 2.0), every)
    for _ in range(2):  # (the second one finds contexts that are no numbers in its cache, too)
        assert np.array_equal(step(lay, broken, dense, 2.0), every)
        out = lay.out.view(B, L, -1)
        assert torch.isnan(lay.c[0]).all() and torch.isnan(out[0]).all()
        assert torch.equal(out[1], well.out.view(B, L, -1)[1])
    # sparse, and mended: rows 0 to 9 of the first sequence, token 3 among them, and what its other rows still hold stays
    few, _, il = _lists(2, B, L, (10, 0), 30)
    few = np.arange(10, dtype=np.int32)
    il.idx[:10] = torch.from_numpy(few).cuda()
    assert np.array_equal(step(lay, x0, il, 0.5), few)
    out = lay.out.view(B, L, -1)
    assert torch.isfinite(out[0, :10]).all() and torch.isnan(out[0, 10:]).all()
    # mended, dense
    for z in (lay, well):
        got = step(z, x1, dense, 2.0)
        assert np.array_equal(got, every)
    assert torch.equal(lay.out, well.out) and torch.equal(lay.c, well.c)
    lay.close(), well.close()
