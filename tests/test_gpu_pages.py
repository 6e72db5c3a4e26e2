"""Requests over pages of keys and values: the page accounting, the pass that writes rows into pages, attention over pages, and all three as a
server runs them, against plain 64-bit forms.

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
THETA, EPS = 10000.0, 1e-5


def say(*a):
    print("[case]", *a, flush=True)


def context(t, H, Hkv, dh, rows=4096):
    return Bd.Context(Bd.LayerCfg(256, H, Hkv, dh, 256, 1, rows, 0, Bd.F32 if t == "f32" else Bd.BF16, EPS, THETA))


def dev(a, t="f32"):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(TD[t])


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def host(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def within(got, want, tol, what):
    got, want = host(got) if torch.is_tensor(got) else got, np.asarray(want)
    assert got.shape == want.shape, what
    assert np.all(np.isfinite(got)), what + ": values that are no numbers"
    bad = np.abs(got - want) > tol
    assert not bad.any(), "%s: %d values off, the worst %.3g of its tolerance" % (what, bad.sum(), np.max(np.abs(got - want) / np.maximum(tol, 1e-300)))


# ---- the page accounting ----------------------------------------------------------------------------------

def plan_in_words(table, free, n_free, length, new, rows, P, cap):
    """dyllm_page_plan, request by request; returns (table, free, n_free, length_out, offsets, pos, slot, whether all fitted)"""
    table, free, R, width = table.copy(), free.copy(), len(length), table.shape[1]
    length, fine = np.clip(length, 0, width * P), True
    unfit = np.maximum(new, 0) > width * P
    new = np.where(unfit, length, np.maximum(new, 0))
    rows = np.clip(rows, 0, new)
    held, need = -(-length // P), -(-new // P)
    back = [table[r, e] for r in range(R) for e in range(need[r], held[r])]
    stack = list(free[:n_free]) + back[::-1]  # (as they are taken)
    served, fits = [], True
    for r in range(R):
        gain = max(need[r] - held[r], 0)
        if gain:
            fits = fits and gain <= len(stack)
            if fits:
                for e in range(held[r], need[r]):
                    table[r, e] = stack.pop()
        served.append((not gain or fits) and not unfit[r])
        fine = fine and served[-1]
    free[n_free:len(stack)] = stack[n_free:][::-1]  # (lost pages that nobody took, in their order)
    offsets = np.concatenate([[0], np.cumsum(rows)])
    pos, slot = [], []
    for r in range(R):
        for i in range(new[r] - rows[r], new[r]):
            pos.append(i)
            slot.append(table[r, i // P] * P + i % P if served[r] else -1)
    fine = fine and offsets[-1] <= cap
    return table, free, len(stack), np.where(served, new, length), np.minimum(offsets, cap), np.array(pos[:cap]), np.array(slot[:cap]), fine


PLANS = [  # requests, page size, longest, room in the pool over what is needed, rows at most, kinds of requests
    (1, 16, 40, 4, 64, "decode"), (1, 64, 0, 0, 8, "decode"), (3, 32, 100, 1, 200, "mixed"), (64, 16, 300, 8, 64, "decode"), (65, 64, 700, 3, 70000, "mixed"),
    (257, 16, 90, -40, 30000, "mixed"), (1000, 128, 2000, 5, 5000, "mixed"), (1025, 16, 60, 0, 60000, "mixed"), (2500, 1024, 9000, -3, 9000, "mixed"),
    (8192, 16, 20, 100, 100000, "mixed"), (50, 16, 64, -1000, 4000, "mixed"), (40, 16, 300, 2, 12000, "ends")]


@pytest.mark.parametrize("R,P,longest,room,cap,kind", PLANS)
def test_plan(R, P, longest, room, cap, kind):
    say("page plan", R, P, longest, room, cap, kind)
    g = W.philox(3, R, P, kind)
    width = -(-max(longest, 1) // P)
    length = g.integers(0, longest + 1, R)
    if kind == "decode":
        new, rows = np.minimum(length + 1, width * P), np.ones(R, np.int64)
    elif kind == "ends":
        new, rows = np.zeros(R, np.int64), np.zeros(R, np.int64)
    else:
        new = np.clip(length + g.integers(-longest, longest + 1, R), 0, longest)
        new[g.random(R) < 0.2] = 0
        same = g.random(R) < 0.2
        new[same] = length[same]
        rows = np.maximum(new - length, 0) + g.integers(0, 5, R) * (g.random(R) < 0.3)
        if R > 10:  # values that are clamped, and a length without room
            length[1], new[2], rows[3], new[4] = -5, -7, 10 ** 6, width * P + 1
    held, need = -(-np.clip(length, 0, width * P) // P), -(-np.clip(new, 0, width * P) // P)
    gain, loss = np.maximum(need - held, 0).sum(), np.maximum(held - need, 0).sum()
    n_free = int(max(gain - loss + room, 0))
    pages = g.permutation(int(held.sum()) + n_free + 3)
    table = np.full((R + 2, width), -77)  # (rows for requests that there are not)
    at = 0
    for r in range(R):
        table[r, :held[r]] = pages[at:at + held[r]]
        at += held[r]
    free = np.full(pages.size, -88)
    free[:n_free] = pages[at:at + n_free]
    ctx = context("bf16", 4, 2, 64, 16)
    k = torch.zeros(pages.size, 1, P, 8, dtype=torch.bfloat16, device="cuda")
    p = Bd.Pages(k, k.clone(), ints(table))
    f, out = ints(free), Bd.PageRows(ints(np.full(R + 1, -99)), ints(np.full(cap, -99)), ints(np.full(cap, -99)))
    len_out, n_out = ints(np.full(R, -99)), ints([-99])
    ins = [ints(length), ints(new), ints(rows), ints([n_free])]
    want = plan_in_words(table[:R], free, n_free, length, new, rows, P, cap)
    for _ in range(2):  # (a repeated call leaves the same)
        ctx.page_plan(p, ins[0], ins[1], ins[2], f, ins[3], out, len_out, n_out)
        torch.cuda.synchronize()
        n = want[4][-1]
        assert np.array_equal(p.table.cpu()[:R], want[0]) and np.all(p.table.cpu().numpy()[R:] == -77)
        assert int(n_out) == want[2] and np.array_equal(f.cpu(), want[1])
        assert np.array_equal(len_out.cpu(), want[3]) and np.array_equal(out.offsets.cpu(), want[4])
        assert np.array_equal(out.pos.cpu()[:n], want[5]) and np.array_equal(out.slot.cpu()[:n], want[6])
        assert np.all(out.pos.cpu().numpy()[n:] == -99) and np.all(out.slot.cpu().numpy()[n:] == -99)
        assert ctx.poll_status() == (0 if want[7] else Bd.ERR_CAPACITY)
    assert all(np.array_equal(x.cpu(), y) for x, y in zip(ins, (length, new, rows, [n_free])))
    ctx.close()


def test_a_pool_stays_whole():
    """Steps of requests that come, grow, fall back and end: no page is ever held twice or lost."""
    say("page plan: many steps")
    g, R, P, width, n_pages = W.philox(5), 37, 16, 12, 150
    ctx = context("bf16", 4, 2, 64, 16)
    p = Bd.Pages.empty(n_pages, 1, P, 8, R, width)
    free, n_free, n_out = ints(g.permutation(n_pages)), ints([n_pages]), ints([0])
    length, len_out = ints(np.zeros(R)), ints(np.zeros(R))
    rows = Bd.PageRows.empty(R * width * P, R)
    short = 0
    for _ in range(60):
        now = length.cpu().numpy()
        new = np.clip(now + g.integers(-40, 60, R), 0, width * P) * (g.random(R) > 0.1)
        ctx.page_plan(p, length, ints(new), ints(np.maximum(new - now, 0)), free, n_free, rows, len_out, n_out)
        short += ctx.poll_status() != 0
        length, len_out, n_free, n_out = len_out, length, n_out, n_free
        held, table = -(-length.cpu().numpy() // P), p.table.cpu().numpy()
        owned = [int(x) for r in range(R) for x in table[r, :held[r]]] + [int(x) for x in free.cpu().numpy()[:int(n_free)]]
        assert sorted(owned) == list(range(n_pages))
    assert 0 < short < 60
    ctx.close()


# ---- norms, rotation on several axes, rows into pages --------------------------------------------------------

def heads(x, g, pos, axis):
    """(y, |n1| + |n2| of every pair) of head vectors x [n, h, dh] at positions pos [axes, n]"""
    dh = x.shape[-1]
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * g if g is not None else x
    a = pos[axis].T * THETA ** (-2.0 * np.arange(dh // 2) / dh)
    co, si = np.cos(a)[:, None], np.sin(a)[:, None]
    n1, n2 = n[..., :dh // 2], n[..., dh // 2:]
    size = np.abs(n1) + np.abs(n2)
    return np.concatenate([n1 * co - n2 * si, n2 * co + n1 * si], -1), np.concatenate([size, size], -1)


def heads_tol(y, size, t):
    # the rounding to the storage type, and in fp32: the sum of squares (19 additions), root, quotient, two products with the gain, cosine and sine
    # (the fraction of a turn 2 pi 2^-32, its rounding, some seven products and sums), two products and a sum: under 64 roundings of the pair's size
    return U[t] * np.abs(y) + 64 * U["f32"] * size + 1e-30


@pytest.mark.parametrize("t,H,Hkv,dh", [("bf16", 4, 4, 64), ("bf16", 6, 2, 128), ("bf16", 32, 32, 128), ("f32", 4, 2, 64), ("f32", 3, 1, 128)])
@pytest.mark.parametrize("gains,pad,axes,P", [("qk", 0, 0, 16), ("q", 8, 1, 64), ("k", 64, 3, 32), ("", 0, 4, 1024)])
def test_heads(t, H, Hkv, dh, gains, pad, axes, P):
    say("head_norm_rope_paged", t, H, Hkv, dh, gains, pad, axes, P)
    g = W.philox(11, t, H, dh, gains)
    ctx = context(t, H, Hkv, dh, 8)  # (no scratch is needed for it)
    width = (H + 2 * Hkv) * dh
    for n, cap in ((0, 3), (1, 1), (300, 333)):
        n_pages = 400 // P + 3
        k0, v0 = (dev(g.standard_normal((n_pages, Hkv, P, dh)), t) for _ in range(2))
        pages = Bd.Pages(k0.clone(), v0.clone(), ints([[0]]))
        slot = g.permutation(n_pages * P)[:cap]
        bad = n > 5
        if bad:
            slot[2], slot[3], slot[4] = -1, -2 ** 31, n_pages * P
        pos = g.integers(0, 100000, (max(axes, 1), cap))
        pos[:, :4] = np.array([0, 1, -3, 2 ** 31 - 1])[:min(cap, 4)]
        axis = g.integers(0, max(axes, 1), dh // 2)
        rows = Bd.PageRows(ints([0, n // 3, n]), ints(pos[0]), ints(slot))
        qkv = dev(3.0 * g.standard_normal((cap, width + pad)), t)[:, :width]
        gq, gk = (dev(1 + 0.2 * g.standard_normal(dh), t) if c in gains else None for c in "qk")
        q_out = torch.full((cap, H, dh), 7.0, dtype=TD[t], device="cuda")
        ctx.head_norm_rope_paged(qkv, gq, gk, rows, pages, q_out, ints(pos) if axes else None, list(axis) if axes else None)
        torch.cuda.synchronize()
        x = host(qkv)[:n].reshape(n, H + 2 * Hkv, dh)
        as_host = lambda z: None if z is None else host(z)  # noqa: E731
        at = pos[:, :n].astype(np.float64)
        y, size = heads(x[:, :H], as_host(gq), at, axis)
        within(q_out[:n], y, heads_tol(y, size, t), "q")
        assert torch.all(q_out[n:] == 7.0)  # rows behind the count stay
        y, size = heads(x[:, H:H + Hkv], as_host(gk), at, axis)
        ok = (slot[:n] >= 0) & (slot[:n] < n_pages * P)
        flat = lambda z: z.transpose(1, 2).reshape(n_pages * P, Hkv, dh)  # noqa: E731
        to = torch.from_numpy(slot[:n][ok]).cuda()
        within(flat(pages.k)[to], y[ok], heads_tol(y, size, t)[ok], "k")
        assert np.array_equal(host(flat(pages.v)[to]), x[ok][:, H + Hkv:])
        rest = torch.ones(n_pages * P, dtype=torch.bool, device="cuda")
        rest[to] = False
        for new, old in ((pages.k, k0), (pages.v, v0)):
            assert torch.equal(flat(new)[rest], flat(old)[rest])
        assert ctx.poll_status() == (Bd.ERR_INVALID_ARG if bad else 0)
    ctx.close()


def test_heads_agree_with_the_table():
    """On one axis, and on three that all hold the same positions, the rotation is that of dyllm_head_norm_rope up to its table's roundings."""
    say("head_norm_rope_paged: the table's rotation")
    t, H, Hkv, dh, L = "f32", 4, 2, 128, 200
    g = W.philox(13)
    ctx = Bd.Context(Bd.LayerCfg(256, H, Hkv, dh, 256, 1, L, 0, Bd.F32, EPS, THETA))
    qkv = dev(g.standard_normal((L, (H + 2 * Hkv) * dh)))
    none = torch.zeros(8, device="cuda")
    k, v = (torch.zeros(1, L, Hkv, dh, device="cuda") for _ in range(2))
    q = torch.zeros(L, H, dh, device="cuda")
    ctx.head_norm_rope(qkv, None, None, None, 1, L, Bd.make_cache(k, v, none, none), q)
    got = []
    for axis_pos in (None, ints(np.tile(np.arange(L), (3, 1)))):
        pages = Bd.Pages.empty(256 // 16, Hkv, 16, dh, 1, 16, TD[t])
        q2 = torch.zeros_like(q)
        ctx.head_norm_rope_paged(qkv, None, None, Bd.PageRows(ints([0, L]), ints(np.arange(L)), ints(np.arange(L))), pages, q2, axis_pos,
                                 bytes(p % 3 for p in range(dh // 2)))
        got.append((q2, pages.k, pages.v))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))
    x = host(qkv).reshape(L, H + 2 * Hkv, dh)
    size = heads(x[:, :H], None, np.arange(L)[None].astype(np.float64), np.zeros(dh // 2, int))[1]
    within(got[0][0], host(q), 16 * U[t] * size, "q")  # (cosine and sine by 2^-24 here, 2^-22 there, four roundings each)
    ctx.close()


# ---- attention over pages -----------------------------------------------------------------------------------

def attend(q, k, v, pos, t, cap=0.0, slopes=None, block=0, prefix=0, doc=None):
    """(rows, tolerances) in 64 bits of rows q [m, H, dh] at positions pos over keys k, v [n, Hkv, dh]"""
    (m, H, dh), (n, Hkv) = q.shape, k.shape[:2]
    u, u32 = U[t], U["f32"]
    out, tol = np.zeros((m, H, dh)), np.zeros((m, H, dh)) + 1e-30
    if n == 0 or m == 0:
        return out.reshape(m, H * dh), tol.reshape(m, H * dh)
    i, j = np.asarray(pos)[:, None], np.arange(n)[None]
    seen = np.ones((m, n), bool)
    if block:
        seen = (j // block <= i // block) | (j < prefix)
    if doc is not None:
        seen &= (doc[i] == doc[j]) & (doc[i] >= 0)
    for h in range(H):
        kb, vb, qb = k[:, h * Hkv // H], v[:, h * Hkv // H], q[:, h]
        s = qb @ kb.T / math.sqrt(dh)
        # A score is off by its sum's roundings (dh products and sums, the scale, the difference to the maximum: under dh + 8 in fp32); capped by
        # those of an exponential, a reciprocal and a multiply-add of the cap's size (under 8, 2^-23 each for the first two); a bias by its
        # product's, the distance's and the sum's.
        ds = (np.abs(qb) @ np.abs(kb).T / math.sqrt(dh)).max(-1, keepdims=True) * (dh + 8) * u32
        if cap:
            s = cap * np.tanh(s / cap)
            ds = ds + 16 * u32 * cap
        if slopes is not None:
            s = s - slopes[h] * np.abs(i - j)
            ds = ds + 4 * u32 * slopes[h] * np.abs(i - j).max(-1, keepdims=True)
        s = np.where(seen, s, -np.inf)
        some = seen.any(-1)
        top = np.where(some, s.max(-1), 0.0)
        p = np.exp(s - top[:, None])
        p /= np.where(some, p.sum(-1), 1.0)[:, None]
        out[:, h] = p @ vb
        # a weight is off by twice the score's error, the exponential (2^-20), the sum, and in bf16 by its own rounding, twice where the sum is over
        # rounded ones
        w = np.expm1(2 * ds) + 2.0 ** -20 + n * u32 + (2 * u if t == "bf16" else 0.0)
        tol[:, h] += w * (p @ np.abs(vb)) * 1.05 + u * np.abs(out[:, h])
    return out.reshape(m, H * dh), tol.reshape(m, H * dh)


def scores_of(kind, H, prefix):
    """(arguments of attend without the prefix, Scores)"""
    kw = dict(cap=7.0) if "cap" in kind else {}
    if "bias" in kind:
        kw["slopes"] = 2.0 ** (-8.0 * (np.arange(H) + 1) / H)
    if "block" in kind:
        kw["block"] = 24
    if "causal" in kind or "prefix" in kind:
        kw["block"] = 1
    s = Bd.Scores(cap=kw.get("cap", 0.0), block=kw.get("block", 0), slopes=dev(kw["slopes"]) if "slopes" in kw else None,
                  prefix=ints(prefix) if "prefix" in kind else None)
    return kw, s


def paged(g, t, Hkv, dh, P, lengths, spare=3):
    """Pages whose unused places hold NaN, and the keys and values of every request."""
    held = [-(-n // P) for n in lengths]
    n_pages, width = sum(held) + spare, max(max(held), 1)
    order, table = g.permutation(n_pages), np.full((len(lengths), width), 10 ** 9)  # (entries behind a length are not looked at)
    k, v = (np.full((n_pages, Hkv, P, dh), np.nan, np.float32) for _ in range(2))
    keys, values, at = [], [], 0
    for r, n in enumerate(lengths):
        table[r, :held[r]] = order[at:at + held[r]]
        at += held[r]
        kk, vv = (host(dev(g.standard_normal((n, Hkv, dh)), t)) for _ in range(2))
        for i in range(n):
            k[table[r, i // P], :, i % P], v[table[r, i // P], :, i % P] = kk[i], vv[i]
        keys.append(kk)
        values.append(vv)
    return Bd.Pages(dev(k, t), dev(v, t), ints(table)), keys, values


def check_paged(seed, t, H, Hkv, dh, P, lengths, counts, kind, cap=None, room=4096, scale=1.5):
    g = W.philox(seed, t, H, dh, kind)
    ctx = context(t, H, Hkv, dh, room)
    pages, keys, values = paged(g, t, Hkv, dh, P, lengths)
    prefix = [n // 3 for n in lengths]
    kw, scores = scores_of(kind, H, prefix)
    off = np.concatenate([[0], np.cumsum(counts)])
    cap = int(off[-1]) if cap is None else cap
    q = dev(scale * g.standard_normal((max(cap, 1), H, dh)), t)
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lengths, counts)] + [np.full(max(cap, 1) - off[-1], 12345)])
    rows = Bd.PageRows(ints(off), ints(pos), ints(np.zeros_like(pos)))
    out = torch.full((max(cap, 1), H * dh), 7.0, dtype=TD[t], device="cuda")
    ctx.paged_attention(q, pages, rows, ints(lengths), out, scores if kind != "none" else None)
    torch.cuda.synchronize()
    for r in range(len(lengths)):
        rr = slice(off[r], off[r + 1])
        want, tol = attend(host(q)[rr], keys[r], values[r], pos[rr], t, prefix=prefix[r] if "prefix" in kind else 0, **kw)
        within(out[rr], want, tol, "request %d" % r)
    assert torch.all(out[off[-1]:] == 7.0)  # rows behind the last request stay
    assert ctx.poll_status() == 0
    ctx.close()


KINDS = ["none", "causal", "block", "prefix", "cap", "bias causal", "cap bias prefix"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("t,H,Hkv,dh,P", [("bf16", 4, 4, 64, 16), ("bf16", 8, 2, 128, 16), ("bf16", 7, 1, 128, 64), ("bf16", 6, 3, 128, 32), ("f32", 4, 2, 64, 16),
                                          ("f32", 2, 2, 128, 128)])
def test_attention_of_ragged_chunks(t, H, Hkv, dh, P, kind):
    """Requests without tokens, with one, with rows for all of their tokens and with none; lengths that end inside pages and tiles."""
    say("paged attention", t, H, Hkv, dh, P, kind)
    check_paged(21, t, H, Hkv, dh, P, [0, 1, 33, 200, 257, 64, 31], [0, 1, 33, 70, 130, 0, 2], kind, cap=250)


@pytest.mark.parametrize("kind", ["causal", "cap bias prefix"])
@pytest.mark.parametrize("t,H,Hkv,dh,P", [("bf16", 32, 32, 128, 16), ("bf16", 28, 4, 128, 64), ("bf16", 8, 2, 64, 32), ("f32", 4, 4, 64, 16)])
def test_attention_of_single_tokens(t, H, Hkv, dh, P, kind):
    """One token a request: key splits of many lengths, the merge of up to 128 of them."""
    say("paged attention, single tokens", t, H, Hkv, dh, P, kind)
    check_paged(22, t, H, Hkv, dh, P, [1, 700, 128, 129, 2500, 0], [1, 1, 1, 1, 1, 0], kind, room=64)


def test_attention_of_one_long_request():
    say("paged attention, one row of 40000 keys")
    check_paged(23, "bf16", 4, 1, 128, 16, [40000], [1], "causal", room=2048)


@pytest.mark.parametrize("t,room", [("bf16", 1), ("bf16", 64), ("f32", 64)])
def test_attention_of_many_requests(t, room):
    """More requests than lanes; a context whose scratch has room for few splits."""
    say("paged attention, 130 requests", t, room)
    g = W.philox(24)
    lengths = [int(x) for x in g.integers(0, 90, 130)]
    check_paged(24, t, 4, 2, 64, 16, lengths, [min(n, 1) for n in lengths], "causal", room=max(room, 130))


@pytest.mark.parametrize("t,H,Hkv,dh,lengths,counts", [
    ("bf16", 4, 4, 64, (2500, 700, 900, 3000), (1, 1, 1, 29)), ("bf16", 28, 4, 128, (4000,) + (300,) * 7, (8,) + (0,) * 7), ("bf16", 2, 2, 128, (5000, 9), (16, 0)),
    ("bf16", 8, 2, 64, (3000, 200, 50), (0, 3, 3)), ("f32", 4, 2, 64, (900, 2500), (19, 1))])
def test_attention_of_a_chunk_beside_single_tokens(t, H, Hkv, dh, lengths, counts):
    """Few rows a request as a mean, but one request has most of them: its tiles are full, and their keys split."""
    say("paged attention, a chunk beside single tokens", t, H, Hkv, dh, counts)
    check_paged(25, t, H, Hkv, dh, 16, list(lengths), list(counts), "causal")


@pytest.mark.parametrize("t,H,rows", [("bf16", 2, 1), ("bf16", 64, 3), ("f32", 2, 2)])
def test_positions_beyond_24_bits(t, H, rows):
    """A request of 2^24 + 5001 tokens, whose pages are few and used over and over: distances between positions that fp32 does not hold."""
    say("paged attention, positions beyond 24 bits", t, H, rows)
    g = W.philox(27, t)
    dh, P, n, held = 64, 1024, 2 ** 24 + 5001, 7
    ctx = context(t, H, 1, dh)
    k, v = (dev(g.standard_normal((held, 1, P, dh)), t) for _ in range(2))
    width = -(-n // P)
    pages = Bd.Pages(k, v, ints((np.arange(width) % held)[None]))
    slopes = np.where(np.arange(H) % 2 == 0, 0.5, 0.25)
    pos = np.arange(n - rows, n)
    q = dev(g.standard_normal((rows, H, dh)), t)
    out = torch.zeros(rows, H * dh, dtype=TD[t], device="cuda")
    ctx.paged_attention(q, pages, Bd.PageRows(ints([0, rows]), ints(pos), ints(np.zeros(rows))), ints([n]), out, Bd.Scores(block=1, slopes=dev(slopes)))
    torch.cuda.synchronize()
    near = np.arange(n - 1500, n)  # (a key further away weighs less than e^(12 - 375) of the nearest ones)
    kk, vv = (host(x)[near // P % held, 0, near % P][:, None] for x in (k, v))
    want, tol = attend(host(q), kk, vv, pos - near[0], t, slopes=slopes, block=1)
    within(out, want, tol, "rows")
    ctx.close()


def test_counts_below_zero():
    """Offsets that no plan leaves: no row is read or written."""
    say("paged attention and heads, a negative count")
    ctx = context("bf16", 2, 1, 64)
    pages = Bd.Pages.empty(4, 1, 16, 64, 2, 2, torch.bfloat16)
    before = pages.k.clone()
    rows = Bd.PageRows(ints([0, 3, -5]), ints([0, 1, 2]), ints([0, 1, 2]))
    q, out = torch.ones(3, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.full((3, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    ctx.head_norm_rope_paged(torch.ones(3, 256, dtype=torch.bfloat16, device="cuda"), None, None, rows, pages, q)
    ctx.paged_attention(q, pages, rows, ints([16, 16]), out)
    torch.cuda.synchronize()
    assert torch.all(q == 1.0) and torch.all(out == 7.0) and torch.equal(pages.k, before)
    ctx.close()


@pytest.mark.parametrize("R", [64, 65, 128, 129, 1100])
@pytest.mark.parametrize("t,H,Hkv,dh", [("bf16", 4, 1, 64), ("bf16", 2, 2, 128), ("f32", 2, 1, 64)])
def test_attention_of_more_requests_than_lanes(t, H, Hkv, dh, R):
    """Requests without rows and without keys among them, runs of such, and a long one that is split."""
    say("paged attention, requests", t, H, Hkv, dh, R)
    g = W.philox(26, R)
    lengths = [int(x) for x in g.integers(0, 40, R)]
    counts = [min(n, int(c)) for n, c in zip(lengths, g.choice([0, 1, 1, 3], R))]
    for i in list(range(10, 50)) + list(range(R - 3, R)):
        counts[i] = 0
    lengths[5], counts[5], lengths[R - 4], counts[R - 4] = 1500, 2, 1100, 40
    check_paged(26, t, H, Hkv, dh, 16, lengths, counts, "causal", cap=sum(counts) + 9)


@pytest.mark.parametrize("H,Hkv", [(24, 24), (10, 5), (16, 8), (12, 3)])
def test_attention_with_every_order_of_heads(H, Hkv):
    """Head counts that the eight dies share in each of the ways; a chunk of some tiles, causal."""
    say("paged attention, heads", H, Hkv)
    check_paged(25, "bf16", H, Hkv, 128, 32, [300, 77], [300, 40], "causal")


def test_large_scores_move_the_reference():
    """Scores of some hundred: the running maximum moves in most tiles."""
    say("paged attention, large scores")
    for counts in ([2], [200]):
        check_paged(26, "bf16", 4, 2, 128, 16, [900], counts, "none", scale=40.0)


def test_entries_that_name_no_page():
    """They are read as the first page and reported; other requests are as they would be."""
    say("paged attention, bad table entries")
    t, H, Hkv, dh, P = "bf16", 8, 2, 128, 16
    for counts in ([1, 1, 1], [90, 150, 3]):
        g, ctx = W.philox(27), context(t, H, Hkv, dh)
        lengths = [100, 200, 50]
        pages, keys, values = paged(g, t, Hkv, dh, P, lengths)
        first = [host(x[0]).transpose(1, 0, 2) for x in (pages.k, pages.v)]
        pages.k[0].nan_to_num_(0.0)
        pages.v[0].nan_to_num_(0.0)
        first = [np.nan_to_num(x) for x in first]
        pages.table[1, 3], pages.table[1, 5] = -1, pages.shape[0]
        for e in (3, 5):
            keys[1][e * P:(e + 1) * P], values[1][e * P:(e + 1) * P] = first
        off = np.concatenate([[0], np.cumsum(counts)])
        pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lengths, counts)])
        q = dev(g.standard_normal((off[-1], H, dh)), t)
        out = torch.zeros(off[-1], H * dh, dtype=TD[t], device="cuda")
        ctx.paged_attention(q, pages, Bd.PageRows(ints(off), ints(pos), ints(pos)), ints(lengths), out, Bd.Scores(block=1))
        assert ctx.poll_status() == Bd.ERR_INVALID_ARG
        for r in range(3):
            rr = slice(off[r], off[r + 1])
            want, tol = attend(host(q)[rr], keys[r], values[r], pos[rr], t, block=1)
            within(out[rr], want, tol, "request %d" % r)
        ctx.close()


def test_lengths_are_clamped_to_the_table():
    say("paged attention, lengths over the table's room")
    g, ctx = W.philox(28), context("bf16", 4, 2, 64)
    pages, keys, values = paged(g, "bf16", 2, 64, 16, [48, 30])
    q, out = dev(g.standard_normal((2, 4, 64)), "bf16"), torch.zeros(2, 256, dtype=torch.bfloat16, device="cuda")
    ctx.paged_attention(q, pages, Bd.PageRows(ints([0, 1, 2]), ints([47, 29]), ints([0, 0])), ints([10 ** 9, -4]), out)
    want, tol = attend(host(q)[:1], keys[0], values[0], [47], "bf16")
    within(out[:1], want, tol, "row 0")
    assert torch.all(out[1] == 0)
    ctx.close()


# ---- a server's steps ---------------------------------------------------------------------------------------

def test_steps_of_a_server():
    """Prompt chunks, then single tokens, then a block that is computed again, through plan, rows into pages and attention, eager and as one captured
    graph that is replayed with eager work of another stream's pool in between; every step against a plain cache."""
    say("a server's steps")
    t, H, Hkv, dh, P, R, width = "bf16", 8, 2, 128, 16, 5, 20
    g = W.philox(31)
    ctx = context(t, H, Hkv, dh, 256)
    cap = 200
    n_pages = 70

    class Server:
        def __init__(self):
            self.pages = Bd.Pages.empty(n_pages, Hkv, P, dh, R, width)
            self.free, self.n_free, self.n_out = ints(g.permutation(n_pages)), ints([n_pages]), ints([0])
            self.length, self.new, self.rows_new, self.len_out = (ints(np.zeros(R)) for _ in range(4))
            self.rows = Bd.PageRows.empty(cap, R)
            self.qkv = torch.zeros(cap, (H + 2 * Hkv) * dh, dtype=TD[t], device="cuda")
            self.q, self.out = torch.zeros(cap, H, dh, dtype=TD[t], device="cuda"), torch.zeros(cap, H * dh, dtype=TD[t], device="cuda")
            self.scores = Bd.Scores(block=8, cap=20.0)

        def step(self):
            ctx.page_plan(self.pages, self.length, self.new, self.rows_new, self.free, self.n_free, self.rows, self.len_out, self.n_out)
            ctx.head_norm_rope_paged(self.qkv, None, None, self.rows, self.pages, self.q)
            ctx.paged_attention(self.q, self.pages, self.rows, self.len_out, self.out, self.scores)
            self.length.copy_(self.len_out)
            self.n_free.copy_(self.n_out)

    eager, replayed = Server(), Server()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        replayed.step()  # (a step of nothing)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            replayed.step()
    torch.cuda.current_stream().wait_stream(side)
    keys, values = [np.zeros((0, Hkv, dh)) for _ in range(R)], [np.zeros((0, Hkv, dh)) for _ in range(R)]
    steps = [([40, 33, 7, 0, 60], None), ([1, 1, 1, 33, 1], None), ([1, 1, 1, 1, 1], None), ([0, 1, 1, 1, 0], 2), ([8, 1, 0, 1, 1], 0), ([1, -20, 1, 8, 1], None),
             ([1, 1, 1, 1, 1], None)]
    for n, (add, again) in enumerate(steps):
        now = np.array([len(x) for x in keys])
        new = np.maximum(now + add, 0)
        rows = np.maximum(add, 0)
        if again is not None:  # a block of a request again
            rows[again] = min(8, new[again])
        off = np.concatenate([[0], np.cumsum(rows)])
        x = dev(g.standard_normal((cap, (H + 2 * Hkv) * dh)), t)
        for server, go in ((replayed, graph.replay), (eager, eager.step)):
            server.new.copy_(ints(new))
            server.rows_new.copy_(ints(rows))
            server.qkv.copy_(x)
            go()
        torch.cuda.synchronize()
        assert ctx.poll_status() == 0
        assert np.array_equal(eager.length.cpu(), new) and np.array_equal(replayed.length.cpu(), new)
        assert torch.equal(eager.out[:off[-1]], replayed.out[:off[-1]]) and int(eager.n_free) == int(replayed.n_free)
        h = host(x).reshape(cap, H + 2 * Hkv, dh)
        for r in range(R):
            rr, pos = slice(off[r], off[r + 1]), np.arange(new[r] - rows[r], new[r])
            y, size = heads(h[rr, H:H + Hkv], None, pos[None].astype(np.float64), np.zeros(dh // 2, int))
            kk, vv = (np.concatenate([z[r], np.zeros((max(new[r] - len(z[r]), 0), Hkv, dh))])[:new[r]] for z in (keys, values))
            at = eager.rows.slot.cpu().numpy()[rr]
            stored = host(eager.pages.k[torch.from_numpy(at // P).cuda(), :, torch.from_numpy(at % P).cuda()]) if len(at) else np.zeros((0, Hkv, dh))
            within(stored, y, heads_tol(y, size, t), "keys of step %d" % n)
            kk[pos], vv[pos] = stored, h[rr, H + Hkv:]
            keys[r], values[r] = kk, vv
            want, tol = attend(host(eager.q)[rr], kk, vv, pos, t, block=8, cap=20.0)
            within(eager.out[rr], want, tol, "step %d, request %d" % (n, r))
    ctx.close()


# ---- refusals -------------------------------------------------------------------------------------------------

def test_what_the_binding_refuses():
    say("refusals")
    ctx = context("bf16", 4, 2, 64, 16)
    p, rows, z = Bd.Pages.empty(4, 2, 16, 64, 2, 3), Bd.PageRows.empty(4, 2), ints([0, 0])
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    q, out, qkv, free, one = bf(4, 4, 64), bf(4, 256), bf(4, 512), ints([0] * 4), ints([0])
    ctx.paged_attention(q, p, rows, z, out)
    ctx.head_norm_rope_paged(qkv, None, None, rows, p, q)
    ctx.page_plan(p, z, z, z, free, one, rows, ints([0, 0]), ints([0]))
    sixteen = bytes(32)
    for call in (
        lambda: Bd.Pages(bf(4, 2, 16, 64), bf(4, 2, 16, 64).float(), p.table), lambda: Bd.Pages(bf(4, 2, 16, 64), bf(4, 2, 16, 64), p.table.long()),
        lambda: Bd.Pages(bf(4, 2, 16, 64), bf(4, 2, 16, 64), p.table.cpu()), lambda: Bd.Pages(bf(4, 2, 16, 64).transpose(1, 2), bf(4, 16, 2, 64), p.table),
        lambda: Bd.PageRows(z, rows.pos, rows.slot[:3]), lambda: Bd.PageRows(z.long(), rows.pos, rows.slot), lambda: Bd.PageRows(ints([0]), rows.pos, rows.slot),
        lambda: Bd.Scores(prefix=z.long()), lambda: Bd.Scores(slopes=bf(4)), lambda: Bd.Scores(doc=z.float()),
        lambda: ctx.paged_attention(q.float(), p, rows, z, out), lambda: ctx.paged_attention(q[:3], p, rows, z, out), lambda: ctx.paged_attention(q, p, rows, z, out[:3]),
        lambda: ctx.paged_attention(q, p, rows, ints([0, 0, 0]), out), lambda: ctx.paged_attention(q, p, rows, z.long(), out),
        lambda: ctx.paged_attention(q, Bd.Pages.empty(4, 1, 16, 64, 2, 3), rows, z, out), lambda: ctx.paged_attention(q, Bd.Pages.empty(4, 2, 16, 64, 1, 3), rows, z, out),
        lambda: ctx.paged_attention(q, Bd.Pages.empty(4, 2, 16, 64, 2, 3, torch.float32), rows, z, out),
        lambda: ctx.paged_attention(q, p, rows, z, out, Bd.Scores(block=1, prefix=one)), lambda: ctx.paged_attention(q, p, rows, z, out, Bd.Scores(slopes=dev([1.0]))),
        lambda: ctx.head_norm_rope_paged(bf(3, 512), None, None, rows, p, q), lambda: ctx.head_norm_rope_paged(bf(4, 448), None, None, rows, p, q),
        lambda: ctx.head_norm_rope_paged(qkv, bf(63), None, rows, p, q), lambda: ctx.head_norm_rope_paged(qkv, None, None, rows, p, q[:3]),
        lambda: ctx.head_norm_rope_paged(qkv, None, None, rows, p, q, ints(np.zeros((2, 3))), sixteen),
        lambda: ctx.head_norm_rope_paged(qkv, None, None, rows, p, q, ints(np.zeros((2, 4))), sixteen[:31]),
        lambda: ctx.head_norm_rope_paged(qkv, None, None, rows, p, q, ints(np.zeros((2, 4)))),
        lambda: ctx.page_plan(p, z, z, one, free, one, rows, ints([0, 0]), ints([0])), lambda: ctx.page_plan(p, z, z, z, free[:3], one, rows, ints([0, 0]), ints([0])),
        lambda: ctx.page_plan(p, z.long(), z, z, free, one, rows, ints([0, 0]), ints([0])),
    ):
        with pytest.raises(ValueError):
            call()

    def refused(code, call):
        with pytest.raises(Bd.DyllmError) as e:
            call()
        assert e.value.code == code
    for size in (8, 24, 2048):
        refused(-3, lambda: ctx.paged_attention(q, Bd.Pages.empty(4, 2, size, 64, 2, 3), rows, z, out))
    refused(-1, lambda: ctx.paged_attention(q, p, rows, z, out, Bd.Scores(cap=-1.0)))
    refused(-1, lambda: ctx.paged_attention(q, p, rows, z, out, Bd.Scores(cap=float("nan"))))
    refused(-1, lambda: ctx.paged_attention(q, p, rows, z, out, Bd.Scores(block=-1)))
    refused(-1, lambda: ctx.page_plan(p, z, z, z, free, one, rows, z, ints([0])))
    refused(-1, lambda: ctx.page_plan(p, z, z, z, free, one, rows, ints([0, 0]), one))
    refused(-1, lambda: ctx.head_norm_rope_paged(qkv, None, None, rows, p, q, ints(np.zeros((2, 4))), bytes([2] * 32)))
    refused(-1, lambda: ctx.head_norm_rope_paged(qkv, None, None, rows, p, q, ints(np.zeros((9, 4))), sixteen))
    refused(-2, lambda: ctx.head_norm_rope_paged(bf(4, 516)[:, :512], None, None, rows, p, q))
    refused(-3, lambda: ctx.paged_attention(q, p, rows, z, out, Bd.Scores(doc=ints([0] * 8))))
    assert ctx.poll_status() == 0
    ctx._dev = 1
    with pytest.raises(ValueError, match="context is on device 1"):
        ctx.paged_attention(q, p, rows, z, out)
    ctx._dev = 0
    ctx.close()
