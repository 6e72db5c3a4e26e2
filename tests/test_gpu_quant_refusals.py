"""What the entry points of normalised heads and of the 8-bit cache refuse of a real context; nothing is launched by these calls."""
import ctypes as C

import pytest
import torch

from paper_2603_08026_amd import binding as Bd

pytestmark = pytest.mark.gpu

B, L, H, HKV, DH, D = 2, 16, 4, 2, 64, 256


@pytest.fixture()
def made():
    ctx = Bd.Context(Bd.LayerCfg(D, H, HKV, DH, 256, B, L, 8, Bd.BF16, 1e-5, 10000.0))
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    rows = Bd.IndexList(torch.tensor([1, 17], dtype=torch.int32, device="cuda"), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"))
    yield ctx, rows, Bd.QuantCache.empty(B, L, HKV, DH), bf
    ctx.close()


def test_tensors_that_do_not_fit(made):
    ctx, rows, c, bf = made
    width = (H + 2 * HKV) * DH
    q, out = bf(2, H, DH), bf(2, H * DH)
    ctx.partial_attention_quant(q, c, rows, B, L, out)
    kv = Bd.make_cache(bf(B, L, HKV, DH), bf(B, L, HKV, DH), bf(8), bf(8))
    short = Bd.IndexList(rows.idx, rows.offsets[:2])
    for call in (
        lambda: ctx.partial_attention_quant(q.float(), c, rows, B, L, out),
        lambda: ctx.partial_attention_quant(bf(1, H, DH), c, rows, B, L, out),
        lambda: ctx.partial_attention_quant(q, c, rows, B, L, out[:1]),
        lambda: ctx.partial_attention_quant(q.cpu(), c, rows, B, L, out),
        lambda: ctx.partial_attention_quant(q, c, short, B, L, out),
        lambda: ctx.partial_attention_quant(q, c, rows, B, L - 1, out),
        lambda: ctx.partial_attention_quant(q, Bd.QuantCache.empty(B, L, HKV + 1, DH), rows, B, L, out),
        lambda: ctx.partial_attention_quant(q, c, None, B, L, out),
        lambda: ctx.partial_attention_quant(q, c, rows, B, L, out, torch.zeros(B, device="cuda")),
        lambda: ctx.partial_attention_quant(q, c, rows, B, L, out, torch.zeros(1, dtype=torch.int32, device="cuda")),
        lambda: ctx.head_norm_rope(bf(2, width - 64), None, None, rows, B, L, kv, q),
        lambda: ctx.head_norm_rope(bf(1, width), None, None, rows, B, L, kv, q),
        lambda: ctx.head_norm_rope(bf(2, 2 * width)[:, ::2], None, None, rows, B, L, kv, q),
        lambda: ctx.head_norm_rope(bf(1, width).expand(2, width), None, None, rows, B, L, kv, q),
        lambda: ctx.head_norm_rope(bf(2, width), bf(DH - 1), None, rows, B, L, kv, q),
        lambda: ctx.head_norm_rope_quant(bf(2, width), None, None, rows, B, L, c, bf(1, H, DH)),
        lambda: ctx.quant_write(bf(1, HKV, DH), bf(2, HKV, DH), rows, B, L, c),
        lambda: ctx.quant_read(c, rows, B, L, bf(2, HKV, DH), bf(1, HKV, DH)),
    ):
        with pytest.raises(ValueError):
            call()


def test_arguments_that_the_library_refuses(made):
    ctx, rows, c, bf = made
    width = (H + 2 * HKV) * DH
    kv = Bd.make_cache(bf(B, L, HKV, DH), bf(B, L, HKV, DH), bf(8), bf(8))
    q = bf(2, H, DH)

    def refused(code, call):
        with pytest.raises(Bd.DyllmError) as e:
            call()
        assert e.value.code == code

    refused(-2, lambda: ctx.head_norm_rope(bf(2, width + 4)[:, :width], None, None, rows, B, L, kv, q))  # rows at no multiple of 16 bytes
    refused(-1, lambda: ctx.head_norm_rope(bf(2 * width + 1)[1:].view(2, width), None, None, rows, B, L, kv, q))
    refused(-1, lambda: ctx.head_norm_rope(bf(2, width), bf(DH + 1)[1:], None, rows, B, L, kv, q))
    big = Bd.IndexList(torch.zeros(9, dtype=torch.int32, device="cuda"), rows.offsets)
    refused(-6, lambda: ctx.quant_write(bf(9, HKV, DH), bf(9, HKV, DH), big, B, L, c))
    odd = Bd.IndexList(rows.idx, torch.zeros(4, dtype=torch.int32, device="cuda"))
    refused(-2, lambda: ctx.quant_read(Bd.QuantCache.empty(3, L, HKV, DH), odd, 3, L, q, q))
    lib, s, z = ctx.lib, C.c_void_p(torch.cuda.current_stream().cuda_stream), C.c_void_p(q.data_ptr())
    r = rows.c()
    bad = Bd.QuantCacheC(c.k.data_ptr(), c.v.data_ptr(), c.k_scale.data_ptr(), c.v_scale.data_ptr(), 2)
    assert lib.dyllm_quant_write(ctx.h, z, z, C.byref(r), B, L, C.byref(bad), s) == -1
    bad = Bd.QuantCacheC(c.k.data_ptr() + 8, c.v.data_ptr(), c.k_scale.data_ptr(), c.v_scale.data_ptr(), 0)
    assert lib.dyllm_partial_attention_quant(ctx.h, z, C.byref(bad), None, C.byref(r), B, L, z, s) == -1
    bad = Bd.QuantCacheC(c.k.data_ptr(), None, c.k_scale.data_ptr(), c.v_scale.data_ptr(), 0)
    assert lib.dyllm_quant_read(ctx.h, C.byref(bad), C.byref(r), B, L, z, z, s) == -1
    assert lib.dyllm_head_norm_rope(ctx.h, z, width - 8, None, None, C.byref(r), B, L, C.byref(kv), z, s) == -2
    x = bf(B * L, D)
    w = Bd.make_weights({n: x for n in ("wq", "wk", "wv", "g_attn")})
    both = (C.byref(kv), C.byref(c.c))
    for a, b in ((None, None), both):
        assert lib.dyllm_qkv_refresh_normed(ctx.h, C.byref(w), None, None, C.c_void_p(x.data_ptr()), C.byref(r), B, L, a, b, z, s) == -1
    assert lib.dyllm_qkv_refresh_normed(ctx.h, C.byref(w), None, None, C.c_void_p(x.data_ptr()), None, B, L, C.byref(kv), None, z, s) == -6
    o = rows.c()  # idx_out is idx_in
    w = Bd.make_weights({n: x for n in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down", "g_attn", "g_ffn")})
    full = Bd.make_cache(x, x, bf(B * L, H * DH), bf(B * L, D))
    assert lib.dyllm_layer_step_quant(ctx.h, C.byref(w), None, None, C.byref(full), C.byref(c.c), None, C.c_void_p(x.data_ptr()), C.byref(r), B, L,
                                      0.5, C.byref(o), None, s) == -1
    alias = Bd.make_cache(x, x, bf(B * L, H * DH), x)
    out = Bd.IndexList.empty(8, B).c()
    assert lib.dyllm_layer_step_quant(ctx.h, C.byref(w), None, None, C.byref(alias), C.byref(c.c), None, C.c_void_p(x.data_ptr()), C.byref(r), B, L,
                                      0.5, C.byref(out), None, s) == -1
    assert ctx.poll_status() == 0


def test_a_context_of_another_device(made, monkeypatch):
    ctx, rows, c, bf = made
    monkeypatch.setattr(ctx, "_dev", 1)
    with pytest.raises(ValueError, match="context is on device 1"):
        ctx.partial_attention_quant(bf(2, H, DH), c, rows, B, L, bf(2, H * DH))
    with pytest.raises(ValueError, match="context is on device 1"):
        ctx.quant_write(bf(2, HKV, DH), bf(2, HKV, DH), rows, B, L, c)
