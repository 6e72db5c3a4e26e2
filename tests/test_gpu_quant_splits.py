"""Attention over the cache in 8 bits where the keys of a sequence are split over workgroups and their results merged, and of lists with room for far
more entries than they hold, against the plain 64-bit form.  (test_quant_host.py checks on the CPU that the cases are planned as they say.)"""
import numpy as np
import pytest
import torch

from synth import workload as W
from tests.test_gpu_quant_cache import TD, _attend, _cache, _check_attend, _ctx, _dev, _host, _lists, _values, _within

pytestmark = pytest.mark.gpu

# type, query heads, KV heads, head_dim, sequences, keys, rows of each sequence -> splits, keys of a split
SPLIT = [
    ("bf16", 2, 1, 128, 6, 6000, 1, 16, 384),
    ("bf16", 4, 2, 64, 6, 6000, 1, 12, 512),
    ("f32", 2, 1, 128, 6, 6000, 1, 16, 384),
    ("f32", 4, 2, 64, 6, 6000, 1, 12, 512),
    ("bf16", 4, 1, 64, 2, 16384, 2, 22, 768),
    ("f32", 2, 1, 128, 2, 16384, 1, 27, 608),
    ("bf16", 8, 2, 128, 1, 32768, 1, 37, 896),
]

# Queries five times as large leave a row a few keys that count, in a split of their own here and there: an error in a split's weight shows.
SHARP = 5.0


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("t,H,Hkv,dh,B,L,rows,splits,chunk", SPLIT)
def test_splits_are_merged(t, H, Hkv, dh, B, L, rows, splits, chunk, codes):
    _check_attend(101, t, H, Hkv, dh, B, L, (rows,) * B, codes, max_rows=rows * B, q_size=SHARP)


# no key; one; a split's; one more; all but one; all -- the splits behind a sequence's last key have none
@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("t,H,Hkv,dh,B,L,rows,splits,chunk", [c for c in SPLIT if c[4] == 6])
def test_splits_of_a_padded_batch(t, H, Hkv, dh, B, L, rows, splits, chunk, codes):
    _check_attend(102, t, H, Hkv, dh, B, L, (rows,) * B, codes, kv_len=(0, 1, chunk, chunk + 1, L - 1, L), max_rows=rows * B, q_size=SHARP)
    _check_attend(103, t, H, Hkv, dh, B, L, (rows,) * B, codes, kv_len=(-1, chunk - 1, 2 * chunk, 3 * chunk + 33, L + 5, 0), max_rows=rows * B, q_size=SHARP)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("t,H,Hkv,dh,B,L,rows,splits,chunk", [c for c in SPLIT if c[4] == 6])
def test_a_vector_that_holds_no_number_in_a_late_split(t, H, Hkv, dh, B, L, rows, splits, chunk, codes):
    """Its sequence and KV head are NaN, every other row is what it was, bit for bit; a query of NaN loses its own row alone."""
    print("[case] splits, nan", t, H, Hkv, dh, codes, flush=True)
    g = W.philox(104, t, dh, codes)
    ctx = _ctx(t, H, Hkv, dh, B, L, rows * B)
    c = _cache(g, B, L, Hkv, dh, codes)
    idx, off, il = _lists(104, B, L, (rows,) * B)
    q = _dev(SHARP * g.standard_normal((idx.size, H, dh)), t)
    good, out = (torch.zeros(idx.size, H * dh, dtype=TD[t], device="cuda") for _ in range(2))
    ctx.partial_attention_quant(q, c, il, B, L, good)
    c.k_scale[1, 0, (splits - 1) * chunk + 3] = float("nan")
    c.v_scale[4, Hkv - 1, (splits - 2) * chunk - 1] = float("nan")
    q[2, H - 1, 5] = float("nan")
    want = np.zeros((idx.size, H), bool)
    group = H // Hkv
    want[1, :group] = want[4, (Hkv - 1) * group:] = want[2, H - 1] = True
    ctx.partial_attention_quant(q, c, il, B, L, out)
    torch.cuda.synchronize()
    o, w = out.view(-1, H, dh), torch.from_numpy(want).cuda()
    lost = torch.isnan(o)
    assert torch.isfinite(good).all()
    assert torch.equal(lost.all(-1), w) and torch.equal(lost.any(-1), w)
    assert torch.equal(o[~w], good.view(-1, H, dh)[~w])
    ctx.close()


def test_split_results_are_the_same_from_run_to_run():
    t, H, Hkv, dh, B, L, rows, splits, chunk = SPLIT[0]
    print("[case] splits, run to run", flush=True)
    g = W.philox(105)
    ctx = _ctx(t, H, Hkv, dh, B, L, rows * B)
    c = _cache(g, B, L, Hkv, dh, "e4m3")
    idx, off, il = _lists(105, B, L, (rows,) * B)
    q = _dev(g.standard_normal((idx.size, H, dh)), t)
    out = [torch.zeros(idx.size, H * dh, dtype=TD[t], device="cuda") for _ in range(3)]
    for o in out:
        ctx.partial_attention_quant(q, c, il, B, L, o)
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])
    ctx.close()


# Lists as a layer hands them on: room for every token, few entries
@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("t,H,Hkv,dh", [("bf16", 4, 2, 128), ("bf16", 6, 1, 64), ("f32", 4, 2, 64), ("f32", 2, 2, 128)])
@pytest.mark.parametrize("B,L,counts", [(1, 3000, (1,)), (1, 900, (90,)), (5, 400, (1, 0, 33, 2, 8)), (70, 60, (1,) * 70), (3, 257, (0, 0, 0))])
def test_attention_of_lists_with_room_for_every_token(B, L, counts, t, H, Hkv, dh, codes):
    _check_attend(106, t, H, Hkv, dh, B, L, counts, codes, cap=B * L, q_size=2.0)
    if B == 5:
        _check_attend(107, t, H, Hkv, dh, B, L, counts, codes, kv_len=(400, 0, 31, 129, 0), cap=B * L, q_size=2.0)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
def test_attention_of_all_tokens_needs_no_room_in_the_context(codes):
    """No list, and a context whose lists hold three entries."""
    t, H, Hkv, dh, B, L = "bf16", 4, 2, 128, 2, 200
    print("[case] attention: all tokens, a small context", codes, flush=True)
    g = W.philox(108, codes)
    ctx = _ctx(t, H, Hkv, dh, B, L, max_rows=3)
    c = _cache(g, B, L, Hkv, dh, codes)
    q = _dev(g.standard_normal((B * L, H, dh)), t)
    out = torch.zeros(B * L, H * dh, dtype=TD[t], device="cuda")
    ctx.partial_attention_quant(q, c, None, B, L, out)
    torch.cuda.synchronize()
    want, tol = _attend(_host(q), _values(c.k, c.k_scale), _values(c.v, c.v_scale), np.array([0, L, 2 * L]), L, None, t)
    _within(out, want, tol, "rows")
    ctx.close()
