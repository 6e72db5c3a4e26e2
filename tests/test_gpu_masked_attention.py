"""Attention rows over a [B, L] cache with masked and reshaped scores, against a plain 64-bit form; what lies in masked places; row lists of every kind."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2603_08026_amd import binding as Bd
from synth import workload as W
from tests.test_gpu_pages import TD, attend, context, dev, host, ints, say, scores_of, within

pytestmark = pytest.mark.gpu

INF = float("inf")


def lists(g, B, L, counts):
    idx = np.concatenate([np.sort(g.choice(L, int(m), replace=False)) + b * L for b, m in enumerate(counts)])
    return idx.astype(np.int64), np.concatenate([[0], np.cumsum(counts)])


def documents(g, B, L, kind):
    if kind == "runs":  # neighbours, with padding at the end
        d = np.sort(g.integers(0, 5, (B, L)), -1)
        d[:, L - L // 9:] = -1
    elif kind == "mixed":  # any order, large and negative numbers
        d = g.choice([-2 ** 31, -1, 0, 7, 2 ** 31 - 1], (B, L))
    elif kind == "one":
        d = np.full((B, L), 3)
    else:  # one token a document
        d = np.tile(np.arange(L), (B, 1))
    return d


def run(ctx, t, q, k, v, idx, off, B, L, scores, kv_len=None, cap=None):
    n, H, dh = q.shape
    cap = n if cap is None else cap
    buf = np.full(max(cap, 1), 0x7fffffff, np.int64)
    buf[:n] = idx
    qd = torch.full((max(cap, 1), H, dh), float("nan"), dtype=TD[t], device="cuda")
    qd[:n] = q
    out = torch.full((max(cap, 1), H * dh), 7.0, dtype=TD[t], device="cuda")
    ctx.partial_attention_masked(qd, k, v, Bd.IndexList(ints(buf)[:cap], ints(off)), B, L, out, scores, None if kv_len is None else ints(kv_len))
    torch.cuda.synchronize()
    assert torch.all(out[n:] == 7.0)  # rows behind the count stay
    return out[:n]


def check(seed, t, H, Hkv, dh, B, L, counts, kind, docs=None, ragged=False, cap=None):
    g = W.philox(seed, t, H, dh, kind, L)
    ctx = context(t, H, Hkv, dh, max(B * L, 4096)) if B == 1 else Bd.Context(Bd.LayerCfg(256, H, Hkv, dh, 256, B, L, 0, Bd.F32 if t == "f32" else Bd.BF16, 1e-5, 1e4))
    k, v = (dev(g.standard_normal((B, L, Hkv, dh)), t) for _ in range(2))
    idx, off = lists(g, B, L, counts)
    q = dev(1.5 * g.standard_normal((len(idx), H, dh)), t)
    prefix = [L // 3 + b for b in range(B)]
    kw, scores = scores_of(kind, H, prefix)
    doc = None if docs is None else documents(g, B, L, docs)
    if doc is not None:
        scores = Bd.Scores(scores.cap, scores.block, scores.prefix, scores.slopes, ints(doc))
    kv_len = [max(0, L - 37 * b - 1) for b in range(B)] if ragged else None
    out = run(ctx, t, q, k, v, idx, off, B, L, scores, kv_len, cap)
    for b in range(B):
        n, rr = L if kv_len is None else kv_len[b], slice(off[b], off[b + 1])
        pos = idx[rr] - b * L
        want, tol = attend(host(q)[rr], host(k)[b, :n], host(v)[b, :n], pos, t, prefix=prefix[b] if "prefix" in kind else 0, doc=None if doc is None else doc[b], **kw)
        within(out[rr], want, tol, "sequence %d" % b)
    assert ctx.poll_status() == 0
    ctx.close()


KINDS = ["none", "causal", "block", "prefix", "cap", "bias", "cap bias prefix"]
SHAPES = [("bf16", 4, 4, 64), ("bf16", 8, 2, 128), ("f32", 4, 2, 64)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("t,H,Hkv,dh", SHAPES)
@pytest.mark.parametrize("counts", [(3, 0, 1), (150, 259, 40)])
def test_rows(t, H, Hkv, dh, kind, counts):
    say("masked attention", t, H, Hkv, dh, kind, counts)
    check(41, t, H, Hkv, dh, 3, 259, counts, kind, ragged=True, cap=sum(counts) + 5)


@pytest.mark.parametrize("docs", ["runs", "mixed", "one", "each"])
@pytest.mark.parametrize("kind", ["none", "prefix", "cap bias causal"])
@pytest.mark.parametrize("t,H,Hkv,dh", SHAPES + [("bf16", 6, 2, 128)])
@pytest.mark.parametrize("counts", [(2, 5), (300, 161)])
def test_documents(t, H, Hkv, dh, kind, docs, counts):
    say("masked attention, documents", t, H, Hkv, dh, kind, docs, counts)
    check(42, t, H, Hkv, dh, 2, 300, counts, kind, docs)


@pytest.mark.parametrize("t,dh", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("counts", [(4,), (120,)])
def test_documents_of_a_padded_batch(t, dh, counts):
    """Documents and a length: rows behind the keys see those of their document that exist."""
    say("masked attention, documents and lengths", t, counts)
    for docs in ("runs", "mixed"):
        g = W.philox(43, t, counts[0])
        B, L, H, Hkv, n = 1, 130, 4, 2, 77
        ctx = context(t, H, Hkv, dh)
        k, v = (dev(g.standard_normal((B, L, Hkv, dh)), t) for _ in range(2))
        idx, off = lists(g, B, L, counts)
        q, doc = dev(1.5 * g.standard_normal((len(idx), H, dh)), t), documents(g, B, L, docs)
        out = run(ctx, t, q, k, v, idx, off, B, L, Bd.Scores(doc=ints(doc)), [n])
        want, tol = attend(host(q), host(k)[0, :n], host(v)[0, :n], idx, t, doc=doc[0])
        within(out, want, tol, docs)
        ctx.close()


def test_key_splits():
    """Few rows of long sequences: several workgroups a row, documents and causal order that leave some of them without keys."""
    say("masked attention, key splits")
    for kind, docs in (("causal", None), ("prefix", None), ("none", "runs"), ("cap bias causal", "mixed")):
        for t, dh in (("bf16", 128), ("bf16", 64), ("f32", 64)):
            check(44, t, 4, 2, dh, 2, 3001, (3, 1), kind, docs)


@pytest.mark.parametrize("t,dh", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_key_splits_of_one_sequence_with_most_rows(t, dh):
    say("masked attention, key splits of full tiles", t, dh)
    check(47, t, 4, 2, dh, 2, 3001, (8, 0), "causal")
    check(47, t, 2, 2, dh, 3, 2000, (1, 21, 2), "prefix")


@pytest.mark.parametrize("t,dh", [("bf16", 64), ("f32", 64)])
def test_more_sequences_than_lanes(t, dh):
    say("masked attention, 70 sequences", t, dh)
    check(48, t, 2, 1, dh, 70, 33, tuple((0, 33, 5, 1)[b % 4] for b in range(70)), "causal")
    check(48, t, 2, 1, dh, 70, 33, tuple((2, 7, 1)[b % 3] for b in range(70)), "block", "runs")


def test_plain_scores_are_those_of_partial_attention():
    """Scores that change nothing: each form within its own tolerance of the other."""
    say("masked attention, nothing masked")
    t, H, Hkv, dh, B, L = "bf16", 8, 2, 128, 2, 300
    g = W.philox(45)
    ctx = Bd.Context(Bd.LayerCfg(256, H, Hkv, dh, 256, B, L, 0, Bd.BF16, 1e-5, 1e4))
    k, v = (dev(g.standard_normal((B, L, Hkv, dh)), t) for _ in range(2))
    for counts in ((3, 2), (200, 300)):
        idx, off = lists(g, B, L, counts)
        q = dev(g.standard_normal((len(idx), H, dh)), t)
        il = Bd.IndexList(ints(idx), ints(off))
        a, b = (torch.zeros(len(idx), H * dh, dtype=TD[t], device="cuda") for _ in range(2))
        ctx.partial_attention(q, k, v, il, B, L, a)
        ctx.partial_attention_masked(q, k, v, il, B, L, b)
        for s in range(2):
            rr = slice(off[s], off[s + 1])
            want, tol = attend(host(q)[rr], host(k)[s], host(v)[s], idx[rr] - s * L, t)
            within(a[rr], want, tol, "partial_attention")
            within(b[rr], want, tol, "partial_attention_masked")
    ctx.close()


def test_all_tokens():
    """rows None is the list of all tokens."""
    say("masked attention, all tokens")
    g = W.philox(46)
    for t, H, Hkv, dh, B, L in (("bf16", 4, 2, 128, 2, 150), ("f32", 4, 4, 64, 3, 33), ("bf16", 2, 2, 64, 1, 1)):
        ctx = Bd.Context(Bd.LayerCfg(256, H, Hkv, dh, 256, B, L, 0, Bd.F32 if t == "f32" else Bd.BF16, 1e-5, 1e4))
        k, v = (dev(g.standard_normal((B, L, Hkv, dh)), t) for _ in range(2))
        q = dev(g.standard_normal((B * L, H, dh)), t)
        a, b = (torch.zeros(B * L, H * dh, dtype=TD[t], device="cuda") for _ in range(2))
        s = Bd.Scores(block=1, cap=9.0)
        ctx.partial_attention_masked(q, k, v, None, B, L, a, s)
        idx, off = np.arange(B * L), np.arange(B + 1) * L
        ctx.partial_attention_masked(q, k, v, Bd.IndexList(ints(idx), ints(off)), B, L, b, s)
        torch.cuda.synchronize()
        assert torch.equal(a, b)
        ctx.close()


@pytest.mark.parametrize("t,dh", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("counts", [(4,), (90,)])
@pytest.mark.parametrize("what", ["causal", "docs", "length"])
def test_no_number_in_a_masked_place(t, dh, counts, what):
    """Keys that do not count have no influence, whatever they hold: the results are those over zeros in their place, bit for bit."""
    say("masked attention, no numbers in masked places", t, dh, counts, what)
    g, B, L, H, Hkv = W.philox(47, t, dh, counts[0]), 1, 200, 4, 2
    ctx = context(t, H, Hkv, dh)
    k, v = (dev(g.standard_normal((B, L, Hkv, dh)), t) for _ in range(2))
    idx = np.sort(g.choice(np.arange(0, 150), counts[0], replace=False))
    off = np.array([0, counts[0]])
    q = dev(g.standard_normal((counts[0], H, dh)), t)
    hidden = np.arange(L) > idx.max()  # from all rows
    doc = np.zeros((B, L), int)
    kv_len, scores = None, Bd.Scores(block=1)
    if what == "docs":  # every third key, among those that count
        hidden = np.arange(L) % 3 == 1
        hidden[idx] = False
        doc[0, hidden] = 1
        scores = Bd.Scores(doc=ints(doc))
    if what == "length":
        kv_len, scores = [int(idx.max()) + 1], None
    at = torch.from_numpy(np.flatnonzero(hidden)).cuda()
    outs = []
    for fill in ((0.0, 0.0, 0.0), (float("nan"), INF, -INF)):
        kk, vv = k.clone(), v.clone()
        for i, x in enumerate(fill):
            kk[0, at[i::3]] = x
            vv[0, at[i::3]] = x
        outs.append(run(ctx, t, q, kk, vv, idx, off, B, L, scores, kv_len))
    assert torch.all(torch.isfinite(outs[0]))
    assert torch.equal(outs[0], outs[1])
    ctx.close()


@pytest.mark.parametrize("t,dh", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("rows", [3, 100])
def test_no_number_that_some_rows_see(t, dh, rows):
    """A value that is no finite number reaches the rows that it counts for, in its column alone, and no other row."""
    say("masked attention, no numbers that some rows see", t, dh, rows)
    g, L, H, Hkv = W.philox(48, t, dh, rows), 128, 2, 1
    ctx = context(t, H, Hkv, dh)
    k, v = (dev(g.standard_normal((1, L, Hkv, dh)), t) for _ in range(2))
    idx = np.sort(g.choice(L, rows, replace=False)) if rows > 3 else np.array([9, 60, 127])
    q = dev(0.3 * g.standard_normal((rows, H, dh)), t)
    clean = run(ctx, t, q, k, v, idx, np.array([0, rows]), 1, L, Bd.Scores(block=1))
    bad = {(10, 3): float("nan"), (61, 5): INF, (62, 7): -INF, (100, 11): INF, (101, 11): -INF, (120, 3): INF}
    for (j, c), x in bad.items():
        v[0, j, 0, c] = x
    out = run(ctx, t, q, k, v, idx, np.array([0, rows]), 1, L, Bd.Scores(block=1)).float().view(rows, H, dh).cpu().numpy()
    want = clean.float().view(rows, H, dh).cpu().numpy().copy()
    for n, i in enumerate(idx):
        for c in range(dh):
            xs = [x for (j, cc), x in bad.items() if cc == c and j <= i]
            if xs:
                want[n, :, c] = sum(xs)
    for a, b in ((np.isnan(out), np.isnan(want)), (out == INF, want == INF), (out == -INF, want == -INF)):
        assert np.array_equal(a, b)
    fine = np.isfinite(want)
    assert np.array_equal(out[fine], want[fine])
    ctx.close()


def test_keys_that_are_no_numbers():
    """A key that counts and is no number makes its rows so; masked ones do not."""
    say("masked attention, a key that is no number")
    g, L, H, dh = W.philox(49), 96, 2, 64
    for t in ("bf16", "f32"):
        ctx = context(t, 4, 2, dh)
        k, v = (dev(g.standard_normal((1, L, 2, dh)), t) for _ in range(2))
        k[0, 50, 0, 1] = float("nan")
        idx = np.arange(40, 60)
        out = run(ctx, t, dev(g.standard_normal((20, 4, dh)), t), k, v, idx, np.array([0, 20]), 1, L, Bd.Scores(block=1)).view(20, 4, dh)
        sees = torch.tensor(idx >= 50).cuda()
        assert torch.all(torch.isnan(out[sees, :2])) and torch.all(torch.isfinite(out[~sees])) and torch.all(torch.isfinite(out[:, 2:]))
        ctx.close()


def test_streams_and_graphs():
    """Calls of two contexts on two streams at once, and a captured call that is replayed with eager work between, against eager results."""
    say("masked attention, streams and graphs")
    t, H, Hkv, dh, B, L = "bf16", 4, 2, 128, 2, 2000
    g = W.philox(50)
    k, v = (dev(g.standard_normal((B, L, Hkv, dh)), t) for _ in range(2))
    made = []
    for counts in ((2, 3), (200, 77)):
        idx, off = lists(g, B, L, counts)
        ctx = Bd.Context(Bd.LayerCfg(256, H, Hkv, dh, 256, B, L, 0, Bd.BF16, 1e-5, 1e4))
        q = dev(g.standard_normal((len(idx), H, dh)), t)
        made.append((ctx, q, Bd.IndexList(ints(idx), ints(off)), torch.zeros(len(idx), H * dh, dtype=TD[t], device="cuda"), torch.cuda.Stream()))
    s = Bd.Scores(block=1, slopes=dev(np.full(H, 0.01)))
    call = lambda m, out: m[0].partial_attention_masked(m[1], k, v, m[2], B, L, out, s)  # noqa: E731
    want = []
    for m in made:
        call(m, m[3])
        want.append(m[3].clone())
    torch.cuda.synchronize()
    for _ in range(5):
        for m in made:
            m[3].zero_()
        torch.cuda.synchronize()
        for m in made:
            with torch.cuda.stream(m[4]):
                call(m, m[3])
        torch.cuda.synchronize()
        assert all(torch.equal(m[3], w) for m, w in zip(made, want))
    graphs = []
    for m in made:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=m[4]):
            call(m, m[3])
        graphs.append(graph)
    other = [torch.zeros_like(m[3]) for m in made]
    for _ in range(4):
        for m, graph, o, w in zip(made, graphs, other, want):
            m[3].zero_()
            graph.replay()
            call(m, o)
            torch.cuda.synchronize()
            assert torch.equal(m[3], w) and torch.equal(o, w)
    for m in made:
        m[0].close()


def test_what_is_refused():
    say("refusals")
    B, L = 2, 16
    ctx = Bd.Context(Bd.LayerCfg(256, 4, 2, 64, 256, B, L, 8, Bd.BF16, 1e-5, 1e4))
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    k, q, out, rows = bf(B, L, 2, 64), bf(2, 4, 64), bf(2, 256), Bd.IndexList(ints([1, 17]), ints([0, 1, 2]))
    ctx.partial_attention_masked(q, k, k, rows, B, L, out)
    for call in (
        lambda: ctx.partial_attention_masked(q.float(), k, k, rows, B, L, out), lambda: ctx.partial_attention_masked(q, k[:1], k, rows, B, L, out),
        lambda: ctx.partial_attention_masked(q, k, k.cpu(), rows, B, L, out), lambda: ctx.partial_attention_masked(q, k, k, rows, B, L, out[:1]),
        lambda: ctx.partial_attention_masked(q, k, k, None, B, L, out), lambda: ctx.partial_attention_masked(q, k, k, rows, B, L, out, None, ints([1])),
        lambda: ctx.partial_attention_masked(q, k, k, rows, B, L, out, Bd.Scores(doc=ints([0] * 31))),
        lambda: ctx.partial_attention_masked(q, k, k, rows, B, L, out, Bd.Scores(block=1, prefix=ints([0]))),
        lambda: ctx.partial_attention_masked(q, k, k, rows, B, L, out, Bd.Scores(slopes=torch.zeros(4))),
    ):
        with pytest.raises(ValueError):
            call()

    def refused(code, call):
        with pytest.raises(Bd.DyllmError) as e:
            call()
        assert e.value.code == code
    refused(-6, lambda: ctx.partial_attention_masked(bf(9, 4, 64), k, k, Bd.IndexList(ints([0] * 9), rows.offsets), B, L, bf(9, 256)))
    ctx.partial_attention_masked(bf(32, 4, 64), k, k, None, B, L, bf(32, 256))  # (all tokens need no room in the context)
    refused(-2, lambda: ctx.partial_attention_masked(q, bf(3, L, 2, 64), bf(3, L, 2, 64), Bd.IndexList(rows.idx, ints([0, 1, 2, 2])), 3, L, out))
    refused(-1, lambda: ctx.partial_attention_masked(q, k, k, rows, B, L, out, Bd.Scores(cap=INF)))
    refused(-1, lambda: ctx.partial_attention_masked(bf(2 * 256 + 1)[1:], k, k, rows, B, L, out))
    assert ctx.lib.dyllm_partial_attention_masked(ctx.h, None, None, None, None, None, B, L, None, None, C.c_void_p(0)) == -1
    assert ctx.poll_status() == 0
    ctx.close()
