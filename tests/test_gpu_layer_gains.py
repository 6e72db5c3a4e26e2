"""A layer that normalises its query and key heads: steps that know no such norms refuse it."""
import pytest
import torch

from paper_2603_08026_amd import binding as Bd
from paper_2603_08026_amd.layer import Layer, Stack
from synth import workload as W
from tests.test_gpu_quant_cache import _dev, _layer, _lists

pytestmark = pytest.mark.gpu

B, L, H, HKV, DH = 2, 24, 4, 2, 64


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("gains", [("g_q", "g_k"), ("g_q",), ("g_k",)])
def test_steps_without_head_norms_refuse_them(t, gains):
    print("[case] gains", t, gains, flush=True)
    s, w = _layer(t, H, HKV, DH, B, L, 141, False)
    plain = {n: z for n, z in w.items() if n not in ("g_q", "g_k")}
    normed = dict(plain, **{n: w[n] for n in gains})
    x = _dev(W.philox(142).standard_normal((B * L, s.hidden)), t)
    lay, il = Layer.from_shape(s, B, L), _lists(1, B, L, (3, 2))[2]
    stack = Stack(s, 2, B, L)
    stack.layers[0].set_weights(plain)
    calls = [lambda: lay.full_step(x), lambda: lay.layer_step(x, il, 0.9), lambda: lay.layer_step_approx(x, il, 0.9)]
    stacked = [lambda: stack.full_step(x), lambda: stack.stack_step(x, il, 0.9), lambda: stack.stack_step_approx(x, il, 0.9),
               lambda: stack.denoise_step(Bd.Schedule(1, 1, 0, 0, 0.9), 0, x, None, None, il)]
    lay.set_weights(normed), stack.layers[1].set_weights(normed)
    for call in calls + stacked:
        with pytest.raises(ValueError, match="head"):
            call()
    torch.cuda.synchronize()
    for z in (lay, *stack.layers):
        assert not z.out.any() and not z.c.any() and not z.k.any()
    lay.set_weights(plain), stack.layers[1].set_weights(plain)
    for call in calls + stacked[:3]:
        call()
    torch.cuda.synchronize()
    assert torch.isfinite(lay.out.float()).all() and lay.out.any() and stack.layers[1].out.any()
    lay.close(), stack.close()


def test_the_pieces_take_the_gains_of_a_layer():
    """What there is for such a layer over caches of the storage type: dyllm_qkv_refresh_normed with the layer's own weights and caches."""
    print("[case] gains, pieces", flush=True)
    s, w = _layer("bf16", H, HKV, DH, B, L, 143, False)
    lay = Layer.from_shape(s, B, L)
    lay.set_weights(w)
    x = _dev(W.philox(144).standard_normal((B * L, s.hidden)), "bf16")
    q = torch.zeros(B * L, H, DH, dtype=torch.bfloat16, device="cuda")
    lay.ctx.qkv_refresh_normed(lay.w, lay.g_q, lay.g_k, x, None, B, L, lay.cache, q)
    torch.cuda.synchronize()
    assert q.any() and lay.k.any() and lay.v.any()
    lay.close()
