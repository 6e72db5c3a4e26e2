"""Projections with biases, head norms and rotation over them (dyllm_qkv_refresh_normed), and the contexts of a layer step over the cache in 8 bits,
against plain 64-bit forms.  (test_quant_host.py checks on the CPU that the projections are planned as PLANS says.)"""
import math

import numpy as np
import pytest
import torch

from paper_2603_08026_amd import binding as Bd
from paper_2603_08026_amd.layer import Layer
from synth import workload as W
from tests.helpers import TOL, assert_close
from tests.test_gpu_quant_cache import (CODES, EPS, TD, U, _attend, _dev, _e4m3, _heads, _heads_tol, _host, _layer, _lists, _scales, _values, _within)

pytestmark = pytest.mark.gpu

# hidden, query heads, KV heads, head_dim, listed rows -> K splits, rows in row tiles, splits of the rows behind them (the device's plan)
PLANS = [
    (2048, 8, 2, 128, 129, 4, 129, 1),
    (2048, 16, 4, 64, 300, 3, 300, 1),
    (2048, 8, 2, 128, 600, 2, 600, 1),
    (2048, 8, 2, 128, 1100, 1, 1100, 1),
    (2048, 16, 8, 128, 2075, 1, 2048, 4),
]
B, L = 3, 900


def _raw(g, t, hidden, H, Hkv, dh):
    """Weights, biases and the signs of an input whose elements are all +-64.  The norm leaves the signs and the gain (64 / sqrt(64^2 + 1e-5) is 1 to
    2^-29); gains are powers of two, weights and biases small multiples of 2^-8: in bf16 operands every sum is exact in fp32, in any order."""
    few = lambda *shape: _dev(g.integers(-8, 9, shape) / 256.0, t)  # noqa: E731
    w = {n: few(rows * dh, hidden) for n, rows in (("wq", H), ("wk", Hkv), ("wv", Hkv))}
    w.update({n: 16 * few(rows * dh) for n, rows in (("bq", H), ("bk", Hkv), ("bv", Hkv))})
    w["g_attn"] = _dev(2.0 ** g.integers(-1, 2, hidden), t)
    sign = np.where(g.standard_normal((B * L, hidden)) < 0, -1.0, 1.0)
    return w, sign


def _packed(w, t):
    out = dict(w)
    for n in ("wq", "wk", "wv") if t == "bf16" else ():
        out[n] = torch.empty_like(w[n])
        Bd.pack_weight(w[n], out[n])
    return out


def _expected(t, w, sign, idx, H, Hkv, dh, gq, gk, bias):
    """(q, k, v) as pairs (value, error before any rounding to a storage type) of the listed rows"""
    x = sign[idx] * _host(w["g_attn"])
    K = x.shape[1]
    out = []
    for m, b, heads, g in (("wq", "bq", H, gq), ("wk", "bk", Hkv, gk), ("wv", "bv", Hkv, None)):
        a = _host(w[m])
        raw, size = x @ a.T, np.abs(x) @ np.abs(a).T
        if bias:
            raw, size = raw + _host(w[b]), size + np.abs(_host(w[b]))
        # fp32: K products and sums, the bias, a few roundings of the norm
        err = (K + 24) * U["f32"] * size * (t == "f32")
        raw, err = raw.reshape(-1, heads, dh), err.reshape(-1, heads, dh)
        if m == "wv":
            out.append((raw, err))
            continue
        y, pair = _heads(raw, g, (idx % L).astype(np.float64))
        # an error of x is scaled by g / rms (and by the norm's own derivative, no larger), and a rotation mixes two elements
        by = 1.0 if g is None else np.abs(g).max() / np.sqrt((raw * raw).mean(-1, keepdims=True) + EPS)
        out.append((y, 4 * by * err.max(-1, keepdims=True) + 64 * U["f32"] * pair))
    return out


def _check_refresh(seed, t, hidden, H, Hkv, dh, count, cap, to, gains, bias):
    print("[case] refresh", t, hidden, H, Hkv, dh, count, cap, to, gains, bias, flush=True)
    g = W.philox(seed, t, H, dh, count)
    ctx = Bd.Context(Bd.LayerCfg(hidden, H, Hkv, dh, 256, B, L, 0, Bd.F32 if t == "f32" else Bd.BF16, EPS, 10000.0))
    w, sign = _raw(g, t, hidden, H, Hkv, dh)
    dev = _packed(w, t)
    if not bias:
        dev = {n: z for n, z in dev.items() if n[0] != "b"}
    gq, gk = (_dev(1 + 0.3 * g.standard_normal(dh), t) if gains else None for _ in range(2))
    part = count // 3
    idx, off, il = _lists(seed, B, L, (count - 2 * part, part, part), cap)
    flat = torch.from_numpy(idx.astype(np.int64)).cuda()
    x = _dev(64.0 * sign, t)
    q = torch.full((il.cap, H, dh), 7.0, dtype=TD[t], device="cuda")
    if to == "cache":
        k, v = (torch.full((B, L, Hkv, dh), 5.0, dtype=TD[t], device="cuda") for _ in range(2))
        none = torch.zeros(8, dtype=TD[t], device="cuda")
        cache = Bd.make_cache(k, v, none, none)
    else:
        cache = Bd.QuantCache.empty(B, L, Hkv, dh, CODES[to])
    ctx.qkv_refresh_normed(Bd.make_weights(dev), gq, gk, x, il, B, L, cache, q)
    torch.cuda.synchronize()
    host = lambda z: None if z is None else _host(z)  # noqa: E731
    (yq, eq), (yk, ek), (yv, ev) = _expected(t, w, sign, idx, H, Hkv, dh, host(gq), host(gk), bias)
    assert np.max(eq) < 0.02 * np.std(yq) and np.max(ek) < 0.02 * np.std(yk)  # (what is allowed is far below what is computed)
    _within(q[:count], yq, U[t] * np.abs(yq) + eq, "q")
    assert torch.all(q[count:] == 7.0)
    rest = torch.ones(B * L, dtype=torch.bool, device="cuda")
    rest[flat] = False
    if to == "cache":
        for got, y, e, what in ((k, yk, ek, "k"), (v, yv, ev, "v")):
            _within(got.view(B * L, Hkv, dh)[flat], y, U[t] * np.abs(y) + e, what)
            assert torch.all(got.view(B * L, Hkv, dh)[rest] == 5.0)
    else:
        for cd, sc, y, e, what in ((cache.k, cache.k_scale, yk, ek, "k"), (cache.v, cache.v_scale, yv, ev, "v")):
            val = _values(cd, sc).reshape(B * L, Hkv, dh)[idx]
            scale = _host(sc)[idx // L, :, idx % L][..., None]
            # half a step of a code
            half = 0.5 * scale * (1 + 2.0 ** -15) if to == "int8" else np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * scale)
            want = _scales(y, to)[..., None]
            assert np.all(np.abs(scale / want - 1) <= (1e-4 if to == "int8" else 1.0)), what  # (e4m3: a largest next to a power's end)
            assert np.all(np.abs(val - y) <= half * (1 + 2.0 ** -20) + 2 * e), what
            assert not cd.view(torch.int8).view(B * L, Hkv, dh)[rest].any()
    ctx.close()


@pytest.mark.parametrize("to", ["cache", "e4m3", "int8"])
@pytest.mark.parametrize("hidden,H,Hkv,dh,count,splits,tiled,tail", PLANS)
def test_refresh_of_rows_that_the_device_plans(hidden, H, Hkv, dh, count, splits, tiled, tail, to):
    _check_refresh(111, "bf16", hidden, H, Hkv, dh, count, 2400, to, True, True)


@pytest.mark.parametrize("gains,bias", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("t,hidden,H,Hkv,dh,count,cap,to", [
    ("bf16", 512, 4, 2, 128, 60, 100, "e4m3"), ("bf16", 512, 8, 4, 64, 230, 250, "cache"), ("bf16", 512, 8, 4, 64, 1, 2700, "int8"),
    ("f32", 256, 4, 2, 64, 77, 90, "int8"), ("f32", 256, 4, 1, 128, 400, 2700, "cache"), ("f32", 256, 4, 2, 64, 3, 3, "e4m3")])
def test_refresh_with_biases(t, hidden, H, Hkv, dh, count, cap, to, gains, bias):
    _check_refresh(112, t, hidden, H, Hkv, dh, count, cap, to, gains, bias)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("gains", [False, True])
@pytest.mark.parametrize("t,H,Hkv,dh", [("bf16", 4, 2, 128), ("bf16", 8, 4, 64), ("f32", 4, 2, 64)])
def test_contexts_and_outputs_of_a_layer_step(t, H, Hkv, dh, gains, codes):
    """A dense step, then a sparse one of a list with room for every token, padded sequences: the contexts are the attention of the step's
    queries over the keys and values that the codes stand for, the outputs what the layer makes of these contexts."""
    Bn, Ln = 3, 150
    print("[case] layer step", t, H, Hkv, dh, gains, codes, flush=True)
    s, w = _layer(t, H, Hkv, dh, Bn, Ln, 121, True)
    for n in ("wq", "wk"):  # scores of a few units, so that rows are no mere averages
        w[n] = (4 * w[n]).astype(np.float32)
    if not gains:
        w.pop("g_q"), w.pop("g_k")
    lay = Layer.from_shape(s, Bn, Ln, codes=codes)
    lay.set_weights(w)
    g = W.philox(122, t, dh)
    x = g.standard_normal((Bn * Ln, s.hidden))
    q = torch.zeros(Bn * Ln, H, dh, dtype=TD[t], device="cuda")
    again = Bd.QuantCache.empty(Bn, Ln, Hkv, dh, CODES[codes])
    w64 = {n: z.astype(np.float64) for n, z in w.items()}
    lens = [150, 64, 131]
    for counts, ln in (((150, 150, 150), None), ((20, 5, 0), lens), ((1, 0, 1), lens)):
        idx, off, il = _lists(123 + counts[0], Bn, Ln, counts, Bn * Ln)
        x[idx] = g.standard_normal((idx.size, s.hidden))
        xd = _dev(x, t)
        before = (lay.c.clone(), lay.out.clone())
        got = lay.layer_step_quant(xd, il, 2.0, kv_len=None if ln is None else torch.tensor(ln, dtype=torch.int32, device="cuda"))
        lay.ctx.qkv_refresh_normed(lay.w, lay.g_q, lay.g_k, xd, il, Bn, Ln, again, q)  # (the step's queries)
        torch.cuda.synchronize()
        assert np.array_equal(lay.read_list(got)[0], idx)
        want, tol = _attend(_host(q)[:idx.size], _values(lay.quant.k, lay.quant.k_scale), _values(lay.quant.v, lay.quant.v_scale), off, Ln, ln, t)
        assert np.max(tol) < 0.15 * np.std(want)
        c, out = lay.c.view(Bn * Ln, -1), lay.out.view(Bn * Ln, -1)
        flat = torch.from_numpy(idx.astype(np.int64)).cuda()
        _within(c[flat], want, tol, "contexts")
        h = _host(xd)[idx] + _host(c[flat]) @ w64["wo"].T
        f = h / np.sqrt((h * h).mean(-1, keepdims=True) + s.rms_eps) * w64["g_ffn"]
        a = f @ w64["w_gate"].T
        y = h + (a / (1 + np.exp(-a)) * (f @ w64["w_up"].T)) @ w64["w_down"].T
        assert_close(_host(out[flat]), y, TOL[t], "outputs")
        rest = torch.ones(Bn * Ln, dtype=torch.bool, device="cuda")
        rest[flat] = False
        for new, old in ((c, before[0]), (out, before[1])):
            assert torch.equal(new[rest], old.view(Bn * Ln, -1)[rest])
    lay.close()
