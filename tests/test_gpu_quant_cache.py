"""Head norms with rotation, the key/value cache in 8 bits and attention over it, against plain 64-bit forms.

Tolerances count roundings (u = half a step relative to the value: bf16 2^-8, fp32 2^-24) and are stated where they are used."""
import math

import numpy as np
import pytest
import torch

from paper_2603_08026_amd import binding as Bd
from synth import workload as W

pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
THETA, EPS = 10000.0, 1e-5


def _say(*a):
    print("[case]", *a, flush=True)


def _ctx(t, H, Hkv, dh, B, L, max_rows=0):
    d = 256
    return Bd.Context(Bd.LayerCfg(d, H, Hkv, dh, 256, B, L, max_rows, Bd.F32 if t == "f32" else Bd.BF16, EPS, THETA))


def _dev(a, t="f32"):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(TD[t])


def _host(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def _lists(seed, B, L, counts, cap=None):
    """(token ids, offsets, IndexList); entries behind the count name no token."""
    idx, off = [], np.zeros(B + 1, np.int32)
    for b in range(B):
        r = np.sort(W.philox(seed, "rows", b).choice(L, size=int(counts[b]), replace=False))
        idx.append(r + b * L)
        off[b + 1] = off[b] + r.size
    idx = np.concatenate(idx).astype(np.int32)
    cap = idx.size if cap is None else cap
    buf = np.full(max(cap, 1), 0x7fffffff, np.int32)
    buf[:idx.size] = idx
    return idx, off, Bd.IndexList(torch.from_numpy(buf).cuda()[:cap], torch.from_numpy(off).cuda())


# ---- the plain forms in 64 bits ---------------------------------------------------------------------------

def _heads(x, g, pos):
    """(y, |n1| + |n2| of every pair) of head vectors x [n, h, dh]"""
    dh = x.shape[-1]
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * g if g is not None else x
    a = pos[:, None] * THETA ** (-2.0 * np.arange(dh // 2) / dh)
    co, si = np.cos(a)[:, None], np.sin(a)[:, None]
    n1, n2 = n[..., :dh // 2], n[..., dh // 2:]
    size = np.abs(n1) + np.abs(n2)
    return np.concatenate([n1 * co - n2 * si, n2 * co + n1 * si], -1), np.concatenate([size, size], -1)


def _heads_tol(y, size, t):
    # the rounding to the storage type, and in fp32: the sum of squares (19 additions), root, quotient, two products with the gain, the table's
    # entries, two products and a sum: under 64 roundings of the pair's size
    return U[t] * np.abs(y) + 64 * U["f32"] * size + 1e-30


def _e4m3(z):
    ulp = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(z), 2.0 ** -6))) - 3)
    return np.rint(z / ulp) * ulp


def _scales(x, codes):
    m = np.maximum(np.abs(x).max(-1), 2.0 ** -100)
    if codes == "int8":
        return m / 127
    f, e = np.frexp(m)
    return 2.0 ** np.maximum(e - 9 + (f > 0.875), -100)


def _values(codes, scale):
    """[B, L, Hkv, dh] codes (device) and [B, Hkv, L] scales -> 64-bit values"""
    return _host(codes) * _host(scale).transpose(0, 2, 1)[..., None]


def _attend(q, k, v, off, L, kv_len, t):
    """(rows, tolerances) of exact attention rows in 64 bits; q [n, H, dh], k and v [B, L, Hkv, dh]"""
    n, H, dh = q.shape
    Hkv, u = k.shape[2], U[t]
    out, tol = np.zeros((n, H, dh)), np.zeros((n, H, dh))
    for b in range(len(off) - 1):
        N = L if kv_len is None else min(max(int(kv_len[b]), 0), L)
        rows = slice(off[b], off[b + 1])
        if N == 0 or off[b] == off[b + 1]:
            continue
        for h in range(H):
            kb, vb, qb = k[b, :N, h * Hkv // H], v[b, :N, h * Hkv // H], q[rows, h]
            s = qb @ kb.T / math.sqrt(dh)
            size = np.abs(qb) @ np.abs(kb).T / math.sqrt(dh)
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[rows, h] = p @ vb
            # (keys and values, or their codes, are exact in bf16.)  A score is off by its sum's roundings (dh products and sums, the
            # scales, the difference to the maximum: under dh + 8 in fp32); a weight by twice that, the exponential (2^-20), and in
            # bf16 by its own rounding, twice where the sum is over rounded ones
            ds = size.max(-1, keepdims=True) * (dh + 8) * U["f32"]
            w = np.expm1(2 * ds) + 2.0 ** -20 + N * U["f32"] + (2 * u if t == "bf16" else 0.0)
            tol[rows, h] = w * (p @ np.abs(vb)) * 1.05 + u * np.abs(out[rows, h]) + 1e-30
    return out.reshape(n, H * dh), tol.reshape(n, H * dh)


def _within(got, want, tol, what):
    got, want = _host(got), np.asarray(want)
    assert got.shape == want.shape, what
    assert np.all(np.isfinite(got)), what + ": values that are no numbers"
    d = np.abs(got - want)
    bad = d > tol
    assert not bad.any(), "%s: %d values off, the worst %.3g of its tolerance" % (what, bad.sum(), np.max(d / np.maximum(tol, 1e-300)))


# ---- norms, rotation, merge -------------------------------------------------------------------------------

SHAPES = [("bf16", 4, 4, 64), ("bf16", 6, 2, 64), ("bf16", 8, 1, 128), ("bf16", 32, 32, 128), ("f32", 4, 2, 64), ("f32", 3, 1, 128)]


@pytest.mark.parametrize("t,H,Hkv,dh", SHAPES)
@pytest.mark.parametrize("gains,pad", [("qk", 0), ("q", 8), ("k", 64), ("", 0)])
def test_head_norm_rope(t, H, Hkv, dh, gains, pad):
    B, L = 3, 257
    _say("head_norm_rope", t, H, Hkv, dh, gains, pad)
    g = W.philox(11, t, H, dh, gains)
    ctx = _ctx(t, H, Hkv, dh, B, L)
    width = (H + 2 * Hkv) * dh
    for counts, cap in (((5, 0, 257), 300), ((1, 0, 0), 1), ((0, 0, 0), 4)):
        idx, off, il = _lists(7, B, L, counts, cap)
        n = idx.size
        buf = _dev(3.0 * g.standard_normal((max(cap, 1), width + pad)), t)
        qkv = buf[:, :width]
        gq, gk = (_dev(1 + 0.2 * g.standard_normal(dh), t) if c in gains else None for c in "qk")
        k0, v0 = (_dev(g.standard_normal((B, L, Hkv, dh)), t) for _ in range(2))
        k, v = k0.clone(), v0.clone()
        none = torch.zeros(8, dtype=TD[t], device="cuda")
        q_out = torch.full((cap, H, dh), 7.0, dtype=TD[t], device="cuda")
        ctx.head_norm_rope(qkv, gq, gk, il, B, L, Bd.make_cache(k, v, none, none), q_out)
        torch.cuda.synchronize()
        x = _host(qkv)[:n].reshape(n, H + 2 * Hkv, dh)
        host = lambda z: None if z is None else _host(z)  # noqa: E731
        pos = (idx % L).astype(np.float64)
        y, size = _heads(x[:, :H], host(gq), pos)
        _within(q_out[:n], y, _heads_tol(y, size, t), "q")
        assert torch.all(q_out[n:] == 7.0)  # rows behind the count stay
        y, size = _heads(x[:, H:H + Hkv], host(gk), pos)
        flat = torch.from_numpy(idx.astype(np.int64)).cuda()
        _within(k.view(B * L, Hkv, dh)[flat], y, _heads_tol(y, size, t), "k")
        assert np.array_equal(_host(v.view(B * L, Hkv, dh)[flat]), x[:, H + Hkv:])
        rest = torch.ones(B * L, dtype=torch.bool, device="cuda")
        rest[flat] = False
        for new, old in ((k, k0), (v, v0)):
            assert torch.equal(new.view(B * L, Hkv, dh)[rest], old.view(B * L, Hkv, dh)[rest])
    ctx.close()


def test_head_norm_rope_of_all_tokens_is_the_full_list():
    t, H, Hkv, dh, B, L = "bf16", 4, 2, 128, 2, 65
    _say("head_norm_rope: rows None")
    g = W.philox(12)
    ctx = _ctx(t, H, Hkv, dh, B, L, max_rows=3)  # (no scratch is needed for it)
    big = _ctx(t, H, Hkv, dh, B, L)
    qkv = _dev(g.standard_normal((B * L, (H + 2 * Hkv) * dh)), t)
    gq = _dev(1 + 0.2 * g.standard_normal(dh), t)
    got = []
    for c, il in ((ctx, None), (big, _lists(1, B, L, (L, L))[2])):
        k, v = (torch.zeros(B, L, Hkv, dh, dtype=TD[t], device="cuda") for _ in range(2))
        q = torch.zeros(B * L, H, dh, dtype=TD[t], device="cuda")
        none = torch.zeros(8, dtype=TD[t], device="cuda")
        c.head_norm_rope(qkv, gq, gq, il, B, L, Bd.make_cache(k, v, none, none), q)
        qc = Bd.QuantCache.empty(B, L, Hkv, dh)
        c.head_norm_rope_quant(qkv, gq, gq, il, B, L, qc, q)
        kb, vb = torch.zeros_like(k), torch.zeros_like(v)
        c.quant_read(qc, il, B, L, kb, vb)
        got.append((q, k, v, qc.k.view(torch.int8), qc.v.view(torch.int8), qc.k_scale, qc.v_scale, kb, vb))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))
    ctx.close(), big.close()


# ---- the cache in 8 bits ----------------------------------------------------------------------------------

@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("t,H,Hkv,dh", SHAPES)
def test_head_norm_rope_quant(t, H, Hkv, dh, codes):
    B, L = 2, 131
    _say("head_norm_rope_quant", t, H, Hkv, dh, codes)
    g = W.philox(21, t, H, dh, codes)
    ctx = _ctx(t, H, Hkv, dh, B, L)
    idx, off, il = _lists(3, B, L, (131, 17), 160)
    n, flat = idx.size, torch.from_numpy(idx.astype(np.int64)).cuda()
    qkv = _dev(3.0 * g.standard_normal((160, (H + 2 * Hkv) * dh)), t)
    gq, gk = (_dev(1 + 0.2 * g.standard_normal(dh), t) for _ in range(2))
    c = Bd.QuantCache.empty(B, L, Hkv, dh, CODES[codes])
    for z in (c.k, c.v):
        z.view(torch.int8).fill_(5)
    c.k_scale.fill_(3.0), c.v_scale.fill_(3.0)
    q_out = torch.zeros(160, H, dh, dtype=TD[t], device="cuda")
    ctx.head_norm_rope_quant(qkv, gq, gk, il, B, L, c, q_out)
    back = [torch.zeros(n, Hkv, dh, dtype=TD[t], device="cuda") for _ in range(2)]
    exact = Bd.IndexList(il.idx[:n], il.offsets)
    ctx.quant_read(c, exact, B, L, *back)
    torch.cuda.synchronize()
    x, pos = _host(qkv)[:n].reshape(n, H + 2 * Hkv, dh), (idx % L).astype(np.float64)
    y, size = _heads(x[:, :H], _host(gq), pos)
    _within(q_out[:n], y, _heads_tol(y, size, t), "q")
    for name, cd, sc, bk, (y, size) in (("k", c.k, c.k_scale, back[0], _heads(x[:, H:H + Hkv], _host(gk), pos)),
                                        ("v", c.v, c.v_scale, back[1], (x[:, H + Hkv:], 0.0 * x[:, H + Hkv:]))):
        slack = 64 * U["f32"] * size  # fp32, as in _heads_tol
        scale = _host(sc)[idx // L, :, idx % L]
        want = _scales(y, codes)
        if codes == "int8":  # two divisions behind the largest magnitude
            assert np.all(np.abs(scale - want) <= 64 * U["f32"] * (size.max(-1) / 127 + want))
        else:  # the power of two, or where the largest lies within its error of 448 the next one
            near = np.abs(y).max(-1) / want
            assert np.all((scale == want) | ((near > 448 * (1 - 1e-5)) & (scale == 2 * want)) | ((near < 224 * (1 + 1e-5)) & (scale == want / 2)))
        val = _values(cd, sc).reshape(B * L, Hkv, dh)[idx]
        # half a step of a code: int8 the scale's half (and the product's roundings), e4m3 2^-4 of the value or half its smallest step
        half = 0.5 * scale[..., None] * (1 + 2.0 ** -15) if codes == "int8" else np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * scale[..., None])
        assert np.all(np.abs(val - y) <= half * (1 + 2.0 ** -20) + 2 * slack), name
        assert np.all(np.abs(_host(bk) - val) <= U[t] * np.abs(val)), name
        rest = np.ones(B * L, bool)
        rest[idx] = False
        assert np.all(cd.view(torch.int8).cpu().numpy().reshape(B * L, Hkv, dh)[rest] == 5)
        assert np.all(_host(sc).transpose(0, 2, 1).reshape(B * L, Hkv)[rest] == 3.0)
    ctx.close()


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("t,Hkv,dh", [("bf16", 4, 128), ("bf16", 2, 64), ("f32", 1, 64), ("f32", 3, 128)])
def test_quant_write_by_its_definition(t, Hkv, dh, codes):
    """Codes and scales bit for bit: the largest magnitude and (e4m3) the quotients are exact, int8 has one rounding to each step."""
    B, L = 2, 70
    _say("quant_write", t, Hkv, dh, codes)
    g = W.philox(31, t, Hkv, dh, codes)
    ctx = _ctx(t, 4 * Hkv, Hkv, dh, B, L)
    idx, off, il = _lists(3, B, L, (33, 12))
    n = idx.size
    x = [g.standard_normal((n, Hkv, dh)) * 2.0 ** g.integers(-12, 12, (n, Hkv, 1)) for _ in range(2)]
    x[0][0] = 0.0                    # nothing but zeros
    x[0][1] = 2.0 ** -110            # below the smallest scale
    x[0][2, :, 0] = 448.0            # a largest one that is the type's
    x[0][3, :, :] = 3.0 * 2.0 ** 100
    x[1][4] *= 0.0
    x[1][4, :, dh - 1] = -1e-3       # one element alone
    if codes == "e4m3":              # ties of the codes, subnormal ones among them
        x[1][5] = 0.0
        x[1][5, :, :6] = [448.0, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 1.0625]
    k, v = _dev(x[0], t), _dev(x[1], t)
    c = Bd.QuantCache.empty(B, L, Hkv, dh, CODES[codes])
    ctx.quant_write(k, v, il, B, L, c)
    torch.cuda.synchronize()
    for src, cd, sc in ((k, c.k, c.k_scale), (v, c.v, c.v_scale)):
        y = src.float().cpu().numpy()
        scale = sc.cpu().numpy()[idx // L, :, idx % L]
        got = _host(cd).reshape(B * L, Hkv, dh)[idx]
        if codes == "int8":
            m = np.maximum(np.abs(y).max(-1), np.float32(2.0 ** -100))
            assert np.array_equal(scale, m / np.float32(127))
            assert np.array_equal(got, np.rint(y * (np.float32(127) / m)[..., None]))
        else:
            assert np.array_equal(scale, _scales(y.astype(np.float64), codes))
            assert np.array_equal(got, _e4m3(y.astype(np.float64) / scale[..., None]))
    # e4m3: what is read back and written again is the same
    if codes == "e4m3":
        kb, vb = torch.zeros_like(k), torch.zeros_like(v)
        ctx.quant_read(c, il, B, L, kb, vb)
        again = Bd.QuantCache.empty(B, L, Hkv, dh)
        ctx.quant_write(kb, vb, il, B, L, again)
        k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
        ctx.quant_read(again, il, B, L, k2, v2)
        torch.cuda.synchronize()
        assert torch.equal(kb, k2) and torch.equal(vb, v2)
    ctx.close()


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_vectors_that_hold_no_number(t, codes):
    """An infinity or NaN makes its own vector NaN and no other; attention rows that meet such a key are NaN, the others as ever."""
    B, L, H, Hkv, dh = 2, 40, 4, 2, 64
    _say("inf and nan", t, codes)
    g = W.philox(41, t, codes)
    ctx = _ctx(t, H, Hkv, dh, B, L)
    k, v = (g.standard_normal((B * L, Hkv, dh)) for _ in range(2))
    k[3, 0, 5], k[7, 1, 63], v[9, 1, 0] = np.inf, np.nan, -np.inf
    kd, vd = _dev(k, t), _dev(v, t)
    c = Bd.QuantCache.empty(B, L, Hkv, dh, CODES[codes])
    ctx.quant_write(kd, vd, None, B, L, c)
    kb, vb = torch.zeros_like(kd), torch.zeros_like(vd)
    ctx.quant_read(c, None, B, L, kb, vb)
    idx, off, il = _lists(5, B, L, (4, 4))
    q = _dev(g.standard_normal((idx.size, H, dh)), t)
    out = torch.zeros(idx.size, H * dh, dtype=TD[t], device="cuda")
    ctx.partial_attention_quant(q, c, il, B, L, out)
    torch.cuda.synchronize()
    for back, bad in ((kb, ((3, 0), (7, 1))), (vb, ((9, 1),))):
        lost = torch.isnan(back).all(-1).cpu().numpy()
        want = np.zeros((B * L, Hkv), bool)
        for r, h in bad:
            want[r, h] = True
        assert np.array_equal(lost, want) and np.array_equal(torch.isnan(back).any(-1).cpu().numpy(), want)
    o = out.view(-1, H, dh)
    assert torch.isnan(o[:4]).all() and torch.isfinite(o[4:]).all()  # (every head of the first sequence meets one)
    ctx.close()


# ---- attention --------------------------------------------------------------------------------------------

def _cache(g, B, L, Hkv, dh, codes, kv_len=None):
    """Random codes and scales; behind kv_len codes and scales that are no numbers."""
    c = Bd.QuantCache.empty(B, L, Hkv, dh, CODES[codes])
    for cd, sc in ((c.k, c.k_scale), (c.v, c.v_scale)):
        x = g.standard_normal((B, L, Hkv, dh)).astype(np.float32)
        s = _scales(x, codes).astype(np.float32)
        z = np.rint(x / s[..., None]) if codes == "int8" else x / s[..., None]
        cd.copy_(torch.from_numpy(z).cuda().to(CODES[codes]))
        sc.copy_(torch.from_numpy(np.ascontiguousarray(s.transpose(0, 2, 1))).cuda())
        if kv_len is not None:
            for b in range(B):
                N = min(max(int(kv_len[b]), 0), L)
                cd.view(torch.int8)[b, N:] = 0x7f
                sc[b, :, N:] = float("nan")
    return c


def _check_attend(seed, t, H, Hkv, dh, B, L, counts, codes, kv_len=None, cap=None, max_rows=0, q_size=1.0):
    _say("attend", t, H, Hkv, dh, "B", B, "L", L, "rows", counts, codes, "kv_len", kv_len, "cap", cap)
    g = W.philox(seed, t, H, Hkv, dh, B, L, codes)
    ctx = _ctx(t, H, Hkv, dh, B, L, max_rows)
    idx, off, il = _lists(seed, B, L, counts, cap)
    n, room = idx.size, il.cap
    c = _cache(g, B, L, Hkv, dh, codes, kv_len)
    q = _dev(q_size * g.standard_normal((room, H, dh)), t)
    out = torch.full((room, H * dh), 7.0, dtype=TD[t], device="cuda")
    ln = None if kv_len is None else torch.tensor(kv_len, dtype=torch.int32, device="cuda")
    ctx.partial_attention_quant(q, c, il, B, L, out, ln)
    torch.cuda.synchronize()
    keep = lambda z: np.nan_to_num(z)  # noqa: E731  (padding, which the rows below never read)
    want, tol = _attend(_host(q)[:n], keep(_values(c.k, c.k_scale)), keep(_values(c.v, c.v_scale)), off, L, kv_len, t)
    _within(out[:n], want, tol, "rows")
    assert torch.all(out[n:] == 7.0)
    ctx.close()


# lengths around a tile's, rows around a block's and a tile's, one row a sequence, sequences without rows
@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("t,H,Hkv,dh", [("bf16", 2, 2, 128), ("bf16", 2, 2, 64), ("bf16", 7, 1, 128), ("bf16", 6, 2, 64),
                                        ("f32", 2, 2, 64), ("f32", 4, 2, 128)])
@pytest.mark.parametrize("L,counts", [(1, (1, 1)), (2, (0, 2)), (31, (1, 31)), (33, (33, 1)), (64, (1, 0)), (129, (32, 64)),
                                      (257, (128, 0)), (300, (1, 1)), (1000, (1, 0)), (520, (129, 65))])
def test_attention(t, H, Hkv, dh, L, counts, codes):
    _check_attend(51, t, H, Hkv, dh, 2, L, counts, codes)


# padded batches: no key, one key, ends inside and at a tile; what lies behind is no number
@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("t,H,Hkv,dh", [("bf16", 4, 4, 128), ("bf16", 8, 2, 64), ("bf16", 14, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("counts", [(1, 1, 1, 1, 1, 1), (40, 3, 0, 100, 17, 64)])
def test_attention_of_a_padded_batch(t, H, Hkv, dh, counts, codes):
    _check_attend(52, t, H, Hkv, dh, 6, 300, counts, codes, kv_len=(300, 0, 1, 128, 129, 999), cap=sum(counts) + 9)


@pytest.mark.parametrize("t,H,Hkv,dh", [("bf16", 4, 4, 128), ("bf16", 8, 2, 64), ("f32", 4, 2, 64)])
def test_attention_of_sequences_without_keys(t, H, Hkv, dh):
    _check_attend(53, t, H, Hkv, dh, 2, 500, (3, 70), "e4m3", kv_len=(0, -4))


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
def test_attention_of_many_rows(codes):
    _check_attend(54, "bf16", 4, 2, 128, 3, 700, (700, 301, 129), codes)
    _check_attend(55, "bf16", 4, 4, 64, 2, 700, (700, 513), codes)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("H,Hkv,dh", [(2, 2, 64), (2, 2, 128), (5, 1, 64), (3, 1, 128)])
def test_attention_of_many_rows_in_fp32(H, Hkv, dh, codes):
    """Enough rows for the form of two rows a workgroup, odd numbers of them, padded sequences."""
    _check_attend(61, "f32", H, Hkv, dh, 4, 301, (301, 129, 300, 251), codes, kv_len=(301, 17, 0, 64), cap=1001)


@pytest.mark.parametrize("q_size", [0.0, 30.0])
def test_attention_of_flat_and_of_sharp_rows(q_size):
    _check_attend(56, "bf16", 4, 4, 128, 2, 900, (20, 130), "e4m3", q_size=q_size)


# Many rows take workgroups of 256 rows (heads of 64: 128), where these outnumber the chip's places in the 32-row form: all rows of many
# sequences, lengths around a tile's and around the turns of its rings, rows that leave waves idle and end inside one
@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("dh,B", [(128, 64), (64, 104)])
@pytest.mark.parametrize("L", [16, 33, 64, 65, 97, 160, 193, 225, 260])
def test_attention_of_all_rows(dh, B, L, codes):
    _check_attend(58, "bf16", 32, 1, dh, B, L, (L,) * B, codes)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("dh,Hkv", [(128, 2), (64, 4)])
def test_attention_of_many_ragged_rows(dh, Hkv, codes):
    """28 heads over 2 or 4, rows of 1 to all of a sequence's tokens, lengths from no key to all."""
    B, L = 32, 300
    g = W.philox(59)
    counts = [300, 1, 0, 290, 19, 55, 73, 128] + [int(n) for n in g.integers(200, 301, B - 8)]
    kv_len = [300, 300, 300, 0, 1, 31, 32, 33, 64, 95, 96, 97] + [int(n) for n in g.integers(0, 301, B - 12)]
    _check_attend(59, "bf16", 28, Hkv, dh, B, L, counts, codes, kv_len=kv_len, cap=sum(counts) + 40)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("dh,B,rows", [(128, 64, 97), (64, 104, 97), (128, 64, 2)])
def test_attention_with_vectors_that_hold_no_number(dh, B, rows, codes):
    """Keys, values and queries that are no numbers make NaN of the rows that meet them and leave the others as they were, in both forms."""
    H, Hkv, L = 32, 1, 97
    _say("attend, inf and nan", dh, B, rows, codes)
    g = W.philox(60, dh, rows, codes)
    ctx = _ctx("bf16", H, Hkv, dh, B, L)
    c = _cache(g, B, L, Hkv, dh, codes)
    idx, off, il = _lists(60, B, L, (rows,) * B)
    q = _dev(g.standard_normal((idx.size, H, dh)), "bf16")
    good, out = (torch.zeros(idx.size, H * dh, dtype=TD["bf16"], device="cuda") for _ in range(2))
    ctx.partial_attention_quant(q, c, il, B, L, good)
    c.k_scale[3, 0, 7] = c.v_scale[5, 0, 96] = float("nan")
    want = np.zeros((idx.size, H), bool)
    want[off[3]:off[4]] = want[off[5]:off[6]] = True
    for b, h, x in ((8, 0, np.inf), (9, 31, np.nan), (B - 1, 17, -np.inf)):
        q[int(off[b + 1]) - 1, h, dh - 1] = x
        want[off[b + 1] - 1, h] = True
    ctx.partial_attention_quant(q, c, il, B, L, out)
    torch.cuda.synchronize()
    lost, o, w = torch.isnan(out.view(-1, H, dh)), out.view(-1, H, dh), torch.from_numpy(want).cuda()
    assert torch.isfinite(good).all()
    assert torch.equal(lost.all(-1), w) and torch.equal(lost.any(-1), w)
    assert torch.equal(o[~w], good.view(-1, H, dh)[~w])
    ctx.close()


def test_attention_of_all_tokens_is_the_full_list():
    t, H, Hkv, dh, B, L = "bf16", 4, 2, 128, 2, 200
    _say("attention: rows None")
    g = W.philox(57)
    ctx = _ctx(t, H, Hkv, dh, B, L)
    c = _cache(g, B, L, Hkv, dh, "e4m3")
    q = _dev(g.standard_normal((B * L, H, dh)), t)
    out = [torch.zeros(B * L, H * dh, dtype=TD[t], device="cuda") for _ in range(2)]
    ctx.partial_attention_quant(q, c, None, B, L, out[0])
    ctx.partial_attention_quant(q, c, _lists(1, B, L, (L, L))[2], B, L, out[1])
    torch.cuda.synchronize()
    assert torch.equal(*out)
    ctx.close()


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_codes_beyond_four_gigabytes(t):
    """The last rows of a cache whose codes pass 2^32 bytes: written, read back, attended over."""
    H, Hkv, dh, B, L = 32, 32, 128, 36, 32768
    _say("offsets past 32 bits", t)
    ctx = _ctx(t, H, Hkv, dh, B, L, max_rows=8)
    c = Bd.QuantCache.empty(B, L, Hkv, dh, torch.int8)
    assert c.k.numel() > 1 << 32
    gen = torch.Generator(device="cuda").manual_seed(1)
    last = B - 1
    for cd, sc in ((c.k, c.k_scale), (c.v, c.v_scale)):
        cd[last] = torch.randint(-127, 128, cd[last].shape, device="cuda", generator=gen, dtype=torch.int8)
        sc[last] = 0.01
    ids = np.array([last * L + 5, last * L + L - 1], np.int32)
    off = np.zeros(B + 1, np.int32)
    off[B] = 2
    il = Bd.IndexList(torch.from_numpy(ids).cuda(), torch.from_numpy(off).cuda())
    new = [torch.randn(2, Hkv, dh, device="cuda", generator=gen).to(TD[t]) for _ in range(2)]
    ctx.quant_write(*new, il, B, L, c)
    back = [torch.zeros_like(z) for z in new]
    ctx.quant_read(c, il, B, L, *back)
    q = torch.randn(2, H, dh, device="cuda", generator=gen).to(TD[t])
    out = torch.zeros(2, H * dh, dtype=TD[t], device="cuda")
    ctx.partial_attention_quant(q, c, il, B, L, out)
    torch.cuda.synchronize()
    for z, bk in zip(new, back):  # half a step of int8, and the rounding of what is read
        m = z.float().abs().amax(-1, keepdim=True)
        assert torch.all((bk.float() - z.float()).abs() <= m * (0.5 / 127 + 2.0 ** -8))
    for h in (0, 31):
        k, v = (cd[last, :, h].double().cpu().numpy() * sc[last, h].double().cpu().numpy()[:, None] for cd, sc in ((c.k, c.k_scale), (c.v, c.v_scale)))
        want, tol = _attend(_host(q)[:, h:h + 1], k[None, :, None], v[None, :, None], np.array([0, 2]), L, None, t)
        _within(out.view(2, H, dh)[:, h], want, tol, "head %d" % h)
    ctx.close()


# ---- a run of them together -------------------------------------------------------------------------------

@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("t,dh,Hkv", [("bf16", 128, 2), ("bf16", 64, 4), ("f32", 64, 2)])
def test_refresh_is_its_pieces(t, dh, Hkv, codes):
    """dyllm_qkv_refresh_normed against the pieces: identity projections make the raw rows the normalised rows of x."""
    H, B, L = 4, 2, 90
    hidden = 128 * ((H + 2 * Hkv) * dh // 128)
    _say("qkv_refresh_normed", t, dh, Hkv, codes)
    g = W.philox(61, t, dh, codes)
    ctx = Bd.Context(Bd.LayerCfg(hidden, H, Hkv, dh, 256, B, L, 0, Bd.F32 if t == "f32" else Bd.BF16, EPS, THETA))
    eye = np.eye(hidden)
    mats = dict(wq=eye[:H * dh], wk=eye[H * dh:(H + Hkv) * dh], wv=eye[(H + Hkv) * dh:(H + 2 * Hkv) * dh])
    wt = {n: _dev(m, t) for n, m in mats.items()}
    if t == "bf16":
        packed = {n: torch.empty_like(m) for n, m in wt.items()}
        for n in wt:
            Bd.pack_weight(wt[n], packed[n])
        wt = packed
    wt["g_attn"] = _dev(1 + 0.1 * g.standard_normal(hidden), t)
    w = Bd.make_weights(wt)
    x = _dev(g.standard_normal((B * L, hidden)), t)
    gq, gk = (_dev(1 + 0.2 * g.standard_normal(dh), t) for _ in range(2))
    idx, off, il = _lists(9, B, L, (41, 3), 60)
    n, flat = idx.size, torch.from_numpy(idx.astype(np.int64)).cuda()
    xs = _host(x)[idx]
    rows = _dev(xs / np.sqrt((xs * xs).mean(-1, keepdims=True) + EPS) * _host(wt["g_attn"]), t)  # (bf16: as the GEMM's operand is rounded)
    raw = torch.zeros(60, (H + 2 * Hkv) * dh, dtype=TD[t], device="cuda")
    raw[:n] = rows
    a, b = (Bd.QuantCache.empty(B, L, Hkv, dh, CODES[codes]) for _ in range(2))
    qa, qb = (torch.zeros(60, H, dh, dtype=TD[t], device="cuda") for _ in range(2))
    ctx.qkv_refresh_normed(w, gq, gk, x, il, B, L, a, qa)
    ctx.head_norm_rope_quant(raw, gq, gk, il, B, L, b, qb)
    k, v = (torch.zeros(B, L, Hkv, dh, dtype=TD[t], device="cuda") for _ in range(2))
    none = torch.zeros(8, dtype=TD[t], device="cuda")
    qc = torch.zeros_like(qa)
    ctx.qkv_refresh_normed(w, gq, gk, x, il, B, L, Bd.make_cache(k, v, none, none), qc)
    torch.cuda.synchronize()
    # the rows of x may be rounded the other way (one step, 2 u), a result likewise (2 u), a code (int8: 1 / 127 of the largest; e4m3 2^-3)
    u = 2 * U[t] + 64 * U["f32"]
    step = 1 / 127 if codes == "int8" else 2.0 ** -3
    assert torch.equal(qa, qc)
    size = lambda z: np.abs(z).max(-1, keepdims=True) + 0 * z  # noqa: E731
    ya = _host(qb)[:n]
    assert np.all(np.abs(_host(qa)[:n] - ya) <= 4 * u * size(ya))
    for za, zb, full in ((_values(a.k, a.k_scale), _values(b.k, b.k_scale), k), (_values(a.v, a.v_scale), _values(b.v, b.v_scale), v)):
        za, zb = za.reshape(B * L, Hkv, dh)[idx], zb.reshape(B * L, Hkv, dh)[idx]
        assert np.all(np.abs(za - zb) <= (step + 4 * u) * size(zb))
        assert np.all(np.abs(za - _host(full.view(B * L, Hkv, dh)[flat])) <= (step / 2 + 2 * u) * size(zb))
    ctx.close()


def _layer(t, H, Hkv, dh, B, L, seed, bias):
    s = W.LayerShape(hidden=256, n_heads=H, n_kv_heads=Hkv, head_dim=dh, ffn=384, dtype=t)
    w = W.make_weights(s, layer=seed, std=0.05)
    g = W.philox(seed, "gains")
    if bias:
        for name, n in (("bq", s.dq), ("bk", s.dkv), ("bv", s.dkv)):
            b = g.standard_normal(n).astype(np.float32) * np.float32(0.1)
            w[name] = W.round_bf16(b) if t == "bf16" else b
    for name in ("g_q", "g_k"):
        b = (1 + 0.2 * g.standard_normal(dh)).astype(np.float32)
        w[name] = W.round_bf16(b) if t == "bf16" else b
    return s, w


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("t,H,Hkv,dh,bias", [("bf16", 4, 2, 128, True), ("bf16", 4, 4, 64, False), ("f32", 4, 2, 64, True)])
def test_layer_step_is_its_pieces(t, H, Hkv, dh, bias, codes):
    """Steps of a layer, dense then sparse with padded sequences: bit for bit what the entry points it is made of leave."""
    from paper_2603_08026_amd.layer import Layer
    B, L = 3, 150
    _say("layer_step_quant", t, H, Hkv, dh, codes)
    s, w = _layer(t, H, Hkv, dh, B, L, 71, bias)
    lay = Layer.from_shape(s, B, L, codes=codes)
    lay.set_weights(w)
    g = W.philox(72, t, dh)
    kv_len = torch.tensor([150, 64, 131], dtype=torch.int32, device="cuda")
    quant = Bd.QuantCache.empty(B, L, Hkv, dh, CODES[codes])
    c, out = torch.zeros_like(lay.c), torch.zeros_like(lay.out)
    cap = B * L
    q = torch.zeros(cap, H, dh, dtype=TD[t], device="cuda")
    ctxr = torch.zeros(cap, H * dh, dtype=TD[t], device="cuda")
    flag, cos = torch.zeros(cap, dtype=torch.uint8, device="cuda"), torch.zeros(cap, device="cuda")
    x = g.standard_normal((B * L, s.hidden))
    steps = [((150, 150, 150), 2.0, None), ((20, 5, 0), 0.9, kv_len), ((0, 0, 0), 0.9, kv_len), ((1, 1, 1), 2.0, kv_len)]
    for i, (counts, tau, ln) in enumerate(steps):
        idx, off, il = _lists(73 + i, B, L, counts, None if i == 0 else 40)
        x[idx] = g.standard_normal((idx.size, s.hidden))
        xd = _dev(x, t)
        got = lay.layer_step_quant(xd, il, tau, kv_len=ln)
        want = Bd.IndexList.empty(cap, B)
        lay.ctx.qkv_refresh_normed(lay.w, lay.g_q, lay.g_k, xd, il, B, L, quant, q)
        lay.ctx.partial_attention_quant(q, quant, il, B, L, ctxr, ln)
        lay.ctx.saliency(ctxr, c, il, B, L, tau, cos, flag, commit=True)
        lay.ctx.compact(flag, il, B, L, want)
        lay.ctx.salient_ffn(lay.w, xd, c, want, B, L, out)
        torch.cuda.synchronize()
        (gi, go), (wi, wo) = lay.read_list(got), lay.read_list(want)
        assert np.array_equal(gi, wi) and np.array_equal(go, wo)
        assert gi.size == (idx.size if tau == 2.0 else gi.size)
        for a, b in ((lay.c, c), (lay.out, out), (lay.quant.k.view(torch.int8), quant.k.view(torch.int8)), (lay.quant.k_scale, quant.k_scale),
                     (lay.quant.v.view(torch.int8), quant.v.view(torch.int8)), (lay.quant.v_scale, quant.v_scale), (lay.cos[:idx.size], cos[:idx.size])):
            assert torch.equal(a, b)
    lay.close()


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_layer_step_stays_near_the_layer_without_codes(t):
    """Without gains a step over int8 codes is dyllm_full_step up to what the codes lose: contexts within the cache's error."""
    from paper_2603_08026_amd.layer import Layer
    B, L, H, Hkv, dh = 2, 96, 4, 2, 64
    _say("layer_step_quant against full_step", t)
    s, w = _layer(t, H, Hkv, dh, B, L, 81, False)
    w.pop("g_q"), w.pop("g_k")
    x = W.philox(82).standard_normal((B * L, s.hidden))
    full, lay = Layer.from_shape(s, B, L), Layer.from_shape(s, B, L, codes="int8")
    for z in (full, lay):
        z.set_weights(w)
    xd = _dev(x, t)
    full.full_step(xd)
    lay.layer_step_quant(xd, _lists(1, B, L, (L, L))[2], 2.0)
    torch.cuda.synchronize()
    a, b = _host(lay.c), _host(full.c)
    # a value is off by half of 1/127 of its head's largest, a score by that share of sum |q k|; a few per cent of the largest context
    k, v = _host(full.k), _host(full.v)
    ds = np.abs(k).max() * 0.5 / 127 * 40.0 / math.sqrt(dh)  # (q of 64 elements about N(0, 1): |q|_1 < 80)
    assert np.max(np.abs(a - b)) <= np.abs(v).max() * (0.5 / 127 + math.expm1(2 * ds) + 4 * U[t])
    full.close(), lay.close()


def test_caches_of_a_layer_go_in_and_out():
    """A layer's caches set from the host are the ones read back, keys and values as the codes hold them; steps that need the other kind of cache are refused."""
    from paper_2603_08026_amd.layer import Layer
    B, L, t, H, Hkv, dh = 2, 50, "bf16", 4, 2, 64
    _say("layer caches")
    s, w = _layer(t, H, Hkv, dh, B, L, 85, False)
    lay, plain = Layer.from_shape(s, B, L, codes="e4m3"), Layer.from_shape(s, B, L)
    for z in (lay, plain):
        z.set_weights(w)
    g = W.philox(86)
    start = {n: g.standard_normal(tuple(getattr(plain, n).shape)) for n in ("k", "v", "c", "out")}
    lay.set_caches(start)
    got = lay.get_caches()
    for n in ("c", "out"):
        assert np.array_equal(got[n], _host(_dev(start[n], t)))
    for n in ("k", "v"):  # half a step of a code, or of its smallest step, of the rounded element
        x = _host(_dev(start[n], t))
        assert np.all(np.abs(got[n] - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * _scales(x, "e4m3")[..., None]))
    lay.set_caches(got)
    again = lay.get_caches()
    assert all(np.array_equal(got[n], again[n]) for n in got)
    x, il = _dev(g.standard_normal((B * L, s.hidden)), t), _lists(1, B, L, (L, L))[2]
    with pytest.raises(ValueError):
        plain.layer_step_quant(x, il, 2.0)
    with pytest.raises(Bd.DyllmError):
        lay.layer_step(x, il, 2.0)
    lay.close(), plain.close()


# ---- streams, graphs --------------------------------------------------------------------------------------

def test_captured_steps_replay():
    """A captured step (one stream, its own inputs), replayed between eager steps of another layer on the same stream, against eager results."""
    from paper_2603_08026_amd.layer import Layer
    B, L, t, H, Hkv, dh = 2, 200, "bf16", 4, 2, 128
    _say("capture and replay")
    s, w = _layer(t, H, Hkv, dh, B, L, 91, True)
    lays = [Layer.from_shape(s, B, L, codes="e4m3") for _ in range(3)]
    for z in lays:
        z.set_weights(w)
    g = W.philox(92)
    xs = [_dev(g.standard_normal((B * L, s.hidden)), t) for _ in range(4)]
    dense, few = _lists(1, B, L, (L, L))[2], _lists(2, B, L, (3, 30))[2]
    kv_len = torch.tensor([200, 77], dtype=torch.int32, device="cuda")
    for z in lays:
        z.layer_step_quant(xs[0], dense, 2.0)
    x = xs[1].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        lays[0].layer_step_quant(x, few, 2.0, kv_len=kv_len)
    for i in (1, 2, 3, 1):
        x.copy_(xs[i])
        graph.replay()
        lays[1].layer_step_quant(xs[i], few, 2.0, kv_len=kv_len)
        torch.cuda.synchronize()
        assert torch.equal(lays[0].c, lays[1].c) and torch.equal(lays[0].out, lays[1].out)
        lays[2].layer_step_quant(xs[i], dense, 2.0)
        torch.cuda.synchronize()
    for z in lays:
        z.close()


def test_on_another_stream():
    t, H, Hkv, dh, B, L = "bf16", 4, 4, 128, 2, 300
    _say("another stream")
    g = W.philox(95)
    ctx = _ctx(t, H, Hkv, dh, B, L)
    c = _cache(g, B, L, Hkv, dh, "e4m3")
    idx, off, il = _lists(4, B, L, (9, 1))
    q = _dev(g.standard_normal((10, H, dh)), t)
    want, got = (torch.zeros(10, H * dh, dtype=TD[t], device="cuda") for _ in range(2))
    ctx.partial_attention_quant(q, c, il, B, L, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx.partial_attention_quant(q, c, il, B, L, got)
    side.synchronize()
    assert torch.equal(got, want)
    ctx.close()
