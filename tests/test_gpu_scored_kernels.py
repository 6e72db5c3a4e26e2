"""Attention with masked and reshaped scores by the kernels for many rows, 128 of bf16 and 32 of fp32 a workgroup, against the plain 64-bit form: every
mask and shape, documents that start and end inside tiles, key splits, pages, values that are no numbers.  (scored_shapes.py says which kernel a shape
is there for, test_scored_plans.py that it gets it.)"""
import numpy as np
import pytest
import torch

from paper_2603_08026_amd import binding as Bd
from synth import workload as W
from tests import scored_shapes as S
from tests.test_gpu_masked_attention import documents, lists, run
from tests.test_gpu_pages import attend, check_paged, dev, host, ints, say, scores_of, within

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
COUNTS = {(2, 800): (449, 351), (2, 461): (300, 161), (2, 1200): (640, 560), (16, 1920): (120,) * 16, (3, 36): (12, 23, 1), (70, 210): (3, 6, 0, 1, 5) * 14,
          (1, 500): (500,), (2, 200): (190, 10), (1, 700): (700,), (1, 800): (800,), (1, 150): (150,)}


def name(s):
    return "-".join(str(x) for x in (s.t, s.H, s.Hkv, s.dh, s.B, s.L, s.cap) + (("split",) if s.split else ()) + (("once",) if s.once else ()))


def parametrized(shapes):
    return pytest.mark.parametrize("s", shapes, ids=name)


def documents_of(g, s, kind):
    if kind == "two":  # the second starts inside a tile, and has most of the tokens
        d = np.tile((np.arange(s.L) >= s.L // 4 + 5).astype(int), (s.B, 1))
    elif kind == "gap":  # padding in the middle, for more rows than a wave has
        d = np.zeros((s.B, s.L), int)
        d[:, s.L // 3:2 * s.L // 3 + 7] = -1
    else:
        d = documents(g, s.B, s.L, kind)
    return d


def context(s):
    return Bd.Context(Bd.LayerCfg(256, s.H, s.Hkv, s.dh, 256, s.B, s.room, 0, Bd.F32 if s.t == "f32" else Bd.BF16, 1e-5, 1e4))


def check(s, kind, docs=None):
    say("many rows", name(s), kind, docs, "lengths" if s.lengths else "")
    g = W.philox(91, s.t, s.H, s.dh, kind, docs or "", s.L)
    ctx = context(s)
    k, v = (dev(g.standard_normal((s.B, s.L, s.Hkv, s.dh)), s.t) for _ in range(2))
    if s.lists:
        idx, off = lists(g, s.B, s.L, COUNTS[s.B, s.cap])
    else:
        idx, off = np.arange(s.B * s.L), np.arange(s.B + 1) * s.L
    q = dev(1.5 * g.standard_normal((s.cap, s.H, s.dh)), s.t)
    prefix = [s.L // 3 + b for b in range(s.B)]
    kw, scores = scores_of(kind, s.H, prefix)
    doc = None if docs is None else documents_of(g, s, docs)
    scores = Bd.Scores(scores.cap, scores.block, scores.prefix, scores.slopes, None if doc is None else ints(doc))
    n = [max(0, s.L - 37 * b - 1) if s.lengths else s.L for b in range(s.B)]

    def call():
        if s.lists:
            return run(ctx, s.t, q, k, v, idx, off, s.B, s.L, scores, n if s.lengths else None)
        out = torch.zeros(s.cap, s.H * s.dh, dtype=q.dtype, device="cuda")
        ctx.partial_attention_masked(q, k, v, None, s.B, s.L, out, scores)
        return out
    out = call()
    hq, hk, hv = host(q), host(k), host(v)
    for b in range(s.B):
        rr = slice(off[b], off[b + 1])
        want, tol = attend(hq[rr], hk[b, :n[b]], hv[b, :n[b]], idx[rr] - b * s.L, s.t, prefix=prefix[b] if "prefix" in kind else 0,
                           doc=None if doc is None else doc[b], **kw)
        within(out[rr], want, tol, "sequence %d" % b)
    assert torch.equal(out, call())  # nothing depends on the order of workgroups
    assert ctx.poll_status() == 0
    ctx.close()


KINDS = ["none", "causal", "block", "prefix", "cap", "bias", "bias causal", "cap bias prefix"]


@pytest.mark.parametrize("kind", KINDS)
@parametrized([S.MANY[0], S.MANY[1], S.MANY[3], S.MANY[4], S.TILE[0], S.TILE[1], S.TILE[2]])
def test_scores(s, kind):
    check(s, kind)


@pytest.mark.parametrize("kind", ["none", "prefix", "cap bias causal"])
@parametrized(S.MANY_LENGTHS + S.TILE_LENGTHS)
def test_lengths(s, kind):
    check(s, kind)


@pytest.mark.parametrize("kind", ["none", "prefix", "cap bias causal"])
@pytest.mark.parametrize("docs", ["runs", "mixed", "one", "each", "two", "gap"])
@parametrized([S.MANY[0], S.MANY[1], S.MANY[3], S.TILE[0], S.TILE[1]])
def test_documents(s, docs, kind):
    check(s, kind, docs)


@pytest.mark.parametrize("docs", ["runs", "mixed", "two", "gap"])
@parametrized([S.MANY[2], S.MANY[4]] + S.MANY_LENGTHS[:2] + S.TILE_LENGTHS)
def test_documents_of_other_shapes(s, docs):
    for kind in ("none", "cap", "bias causal"):
        check(s, kind, docs)


@parametrized(S.MANY_ALL + S.TILE_ALL)
def test_all_tokens(s):
    for kind, docs in (("causal", None), ("none", "two"), ("cap bias prefix", "runs")):
        check(s, kind, docs)


@parametrized(S.MANY_SPLIT + S.TILE_SPLIT)
def test_key_splits(s):
    for kind, docs in (("none", None), ("causal", None), ("cap bias prefix", None), ("none", "two"), ("none", "runs"), ("prefix", "mixed"), ("cap bias causal", "gap")):
        check(s, kind, docs)


PAGES = {(3, 800): ([512, 300, 77], [470, 290, 40]), (3, 500): ([512, 300, 7], [300, 199, 1]), (3, 1200): ([704, 500, 31], [700, 480, 20]),
         (8, 600): ([320, 100, 0, 33, 211, 64, 320, 1], [150, 100, 0, 30, 100, 64, 155, 1]), (4, 460): ([384, 257, 200, 31], [200, 130, 128, 2]),
         (3, 60): ([2048, 700, 33], [40, 19, 1])}


@pytest.mark.parametrize("kind", ["none", "causal", "block", "prefix", "cap", "bias causal", "cap bias prefix"])
@pytest.mark.parametrize("P", [16, 64])
@parametrized(S.MANY_PAGES + S.TILE_PAGES)
def test_pages(s, P, kind):
    say("many rows over pages", name(s), P, kind)
    lengths, counts = PAGES[s.B, s.cap]
    assert -(-max(lengths) // P) * P == s.L
    check_paged(92, s.t, s.H, s.Hkv, s.dh, P, lengths, counts, kind, cap=s.cap, room=s.room)


@pytest.mark.parametrize("kind", ["causal", "cap bias prefix"])
@parametrized(S.TILE_PAGES)
def test_large_pages(s, kind):
    say("many rows over pages of 128", name(s), kind)
    lengths, counts = PAGES[s.B, s.cap]
    check_paged(93, s.t, s.H, s.Hkv, s.dh, 128, lengths, counts, kind, cap=s.cap, room=s.room)


# ---- values that are no numbers ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("what", ["causal", "length", "docs", "docs cap bias causal", "two", "two cap causal"])
@parametrized(S.NO_NUMBER)
def test_no_number_in_a_masked_place(s, what):
    """Keys that do not count have no influence, whatever they hold: the results are those over zeros in their place, bit for bit."""
    say("many rows, no numbers in masked places", name(s), what)
    g = W.philox(94, s.t, s.dh, what)
    ctx = context(s)
    k, v = (dev(g.standard_normal((1, s.L, s.Hkv, s.dh)), s.t) for _ in range(2))
    first = s.L // 8 + 3 if "two" in what else 0
    idx = np.sort(g.choice(np.arange(first, s.L if "docs" in what or "two" in what else s.L - 40), s.cap, replace=False))
    q = dev(g.standard_normal((s.cap, s.H, s.dh)), s.t)
    _, scores = scores_of(what, s.H, None)
    j, doc, kv_len = np.arange(s.L), None, None
    hidden = j > idx.max()
    if "docs" in what:  # every third of the keys that are no rows'
        hidden = (j % 3 == 1) & ~np.isin(j, idx)
        doc = hidden.astype(int)
    elif "two" in what:
        hidden = j < first
        doc = np.where(hidden, 5, 7)
    elif what == "length":
        kv_len = [int(idx.max()) + 1]
    assert hidden.sum() >= 9
    scores = Bd.Scores(scores.cap, scores.block, None, scores.slopes, None if doc is None else ints(doc[None]))
    at, outs = torch.from_numpy(np.flatnonzero(hidden)).cuda(), []
    for fill in ((0.0, 0.0, 0.0), (NAN, INF, -INF)):
        kk, vv = k.clone(), v.clone()
        for n, x in enumerate(fill):
            kk[0, at[n::3]] = x
            vv[0, at[n::3]] = x
        outs.append(run(ctx, s.t, q, kk, vv, idx, np.array([0, s.cap]), 1, s.L, scores, kv_len))
    assert torch.all(torch.isfinite(outs[0]))
    assert torch.equal(outs[0], outs[1])
    ctx.close()


@pytest.mark.parametrize("what", ["causal", "block", "cap causal", "docs causal", "docs cap bias causal"])
@parametrized(S.NO_NUMBER)
def test_no_number_that_some_rows_see(s, what):
    """A value that is no finite number reaches the rows that it counts for, in its column alone, and no other row."""
    say("many rows, no numbers that some rows see", name(s), what)
    g = W.philox(95, s.t, s.dh, what)
    ctx = context(s)
    k, v = (dev(g.standard_normal((1, s.L, s.Hkv, s.dh)), s.t) for _ in range(2))
    idx = np.sort(g.choice(s.L, s.cap, replace=False))
    q = dev(0.3 * g.standard_normal((s.cap, s.H, s.dh)), s.t)
    kw, scores = scores_of(what, s.H, None)
    j = np.arange(s.L)
    doc = (j >= s.L // 3 + 5).astype(int) if "docs" in what else np.zeros(s.L, int)
    # (slopes of a hundredth: no weight is too small for an fp32 number)
    slopes = dev(np.full(s.H, 0.01)) if "bias" in what else None
    scores = Bd.Scores(scores.cap, scores.block, None, slopes, ints(doc[None]) if "docs" in what else None)
    call = lambda: run(ctx, s.t, q, k, v, idx, np.array([0, s.cap]), 1, s.L, scores)  # noqa: E731
    clean = call()
    bad = {(10, 3): NAN, (61, 5): INF, (62, 7): -INF, (s.L // 2, 11): INF, (s.L // 2 + 1, 11): -INF, (s.L - 30, 3): INF, (s.L - 31, 9): -INF, (s.L - 1, 2): NAN}
    for (n, c), x in bad.items():
        v[0, n, :, c] = x
    out = call().float().view(s.cap, s.H, s.dh).cpu().numpy()
    want = clean.float().view(s.cap, s.H, s.dh).cpu().numpy().copy()
    block = kw["block"]
    for n, i in enumerate(idx):
        for c in range(s.dh):
            xs = [x for (jj, cc), x in bad.items() if cc == c and jj // block <= i // block and doc[jj] == doc[i]]
            if xs:
                want[n, :, c] = sum(xs)
    for a, b in ((np.isnan(out), np.isnan(want)), (out == INF, want == INF), (out == -INF, want == -INF)):
        assert np.array_equal(a, b)
    fine = np.isfinite(want)
    assert np.array_equal(out[fine], want[fine])
    ctx.close()
