"""Requests over pages, and attention with shaped scores, where sums of pages and rows pass 2^30 and tensors 2^32 bytes."""
import numpy as np
import pytest
import torch

from paper_2603_08026_amd import binding as Bd
from synth import workload as W
from tests.test_gpu_pages import TD, attend, context, dev, heads, heads_tol, host, ints, say, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("greedy,width", [(16, 2 ** 26), (2048, 2 ** 19)])
def test_gains_beyond_30_bits(greedy, width):
    """Requests that ask for 2^30 pages together, then one that asks for one page, one that gives a page back, one that stays: none behind the first that
    does not fit gains anything, and all others go on."""
    say("page plan: gains of 2^30 pages", greedy, width)
    P, n_pages = 16, 9
    R = 1 + greedy + 3
    ctx = context("bf16", 4, 2, 64, 16)
    k = torch.zeros(n_pages, 1, P, 8, dtype=torch.bfloat16, device="cuda")
    table = torch.full((R, width), -77, dtype=torch.int32, device="cuda")
    table[0, 0], table[R - 2, 0], table[R - 2, 1], table[R - 1, 0] = 4, 5, 6, 7
    length, new, rows = np.zeros(R, int), np.full(R, width * P), np.ones(R, int)
    length[[0, R - 2, R - 1]] = 10, 20, 9
    new[[0, R - 3, R - 2, R - 1]] = 20, 16, 16, 9
    out = Bd.PageRows(*(ints(np.full(n, -99)) for n in (R + 1, R, R)))
    free, len_out, n_out = ints([0, 1, 2] + [-88] * 6), ints(np.full(R, -99)), ints([-99])
    pages = Bd.Pages(k, k.clone(), table)
    for _ in range(2):  # (a repeated call leaves the same)
        ctx.page_plan(pages, ints(length), ints(new), ints(rows), free, ints([3]), out, len_out, n_out)
        assert ctx.poll_status() == Bd.ERR_CAPACITY
        # request 0 takes the lost page 6; the pool is as before
        want = length.copy()
        want[[0, R - 2]] = 20, 16
        assert np.array_equal(len_out.cpu(), want) and int(n_out) == 3
        assert np.array_equal(free.cpu(), [0, 1, 2] + [-88] * 6)
        slot = np.full(R, -1)
        slot[[0, R - 2, R - 1]] = 6 * P + 3, 5 * P + 15, 7 * P + 8
        assert np.array_equal(out.slot.cpu(), slot)
        assert np.array_equal(out.pos.cpu(), new - 1) and np.array_equal(out.offsets.cpu(), np.arange(R + 1))
        assert table[0, :3].tolist() == [4, 6, -77] and table[R - 2, :3].tolist() == [5, 6, -77] and table[R - 1, :2].tolist() == [7, -77]
        assert not torch.any(table[1:R - 2] != -77)
    ctx.close()


def test_lengths_of_more_pages_than_there_are():
    """Lengths that claim 2^30 pages, more than a pool can have: what is given back in excess is dropped, and nothing outside the lists is touched."""
    say("page plan: losses of 2^30 pages")
    P, n_pages, width, R = 16, 6, 2 ** 26, 18
    ctx = context("bf16", 4, 2, 64, 16)
    k = torch.zeros(n_pages, 1, P, 8, dtype=torch.bfloat16, device="cuda")
    table = torch.full((R, width), 3, dtype=torch.int32, device="cuda")
    length, new = np.full(R, width * P), np.zeros(R, int)
    length[R - 1], new[R - 1] = 0, 16
    out = Bd.PageRows(*(ints(np.full(n, -99)) for n in (R + 1, R, R)))
    guard = ints(np.full(n_pages + 64, -88))
    len_out, n_out = ints(np.full(R, -99)), ints([-99])
    ctx.page_plan(Bd.Pages(k, k.clone(), table), ints(length), ints(new), ints(new > 0), guard[:n_pages], ints([0]), out, len_out, n_out)
    torch.cuda.synchronize()
    assert np.array_equal(len_out.cpu(), new) and int(n_out) == n_pages
    assert np.array_equal(guard.cpu(), [3] * n_pages + [-88] * 64) and int(out.slot[0]) == 3 * P + 15
    ctx.poll_status()
    ctx.close()


def test_rows_beyond_30_bits():
    """As many rows as a capacity may have, beside the pages that they take: every output is there."""
    say("page plan: 2^30 rows")
    P, each, R = 1024, 2 ** 29, 3
    cap, n_pages, width = 2 * each, 2 * each // P + 1, each // P
    ctx = context("bf16", 4, 2, 64, 16)
    none = torch.zeros(n_pages, 1, P, 0, dtype=torch.bfloat16, device="cuda")  # (the plan looks at no key)
    pages = Bd.Pages(none, none, torch.full((R, width), -77, dtype=torch.int32, device="cuda"))
    rows = Bd.PageRows(ints([-99] * (R + 1)), *(torch.full((cap,), -99, dtype=torch.int32, device="cuda") for _ in range(2)))
    len_out, n_out = ints([-99] * R), ints([-99])
    free = torch.arange(n_pages, dtype=torch.int32, device="cuda")
    ctx.page_plan(pages, ints([0] * R), ints([each, each, 1]), ints([each, each, 0]), free, ints([n_pages]), rows, len_out, n_out)
    assert ctx.poll_status() == 0
    assert len_out.tolist() == [each, each, 1] and int(n_out) == 0 and rows.offsets.tolist() == [0, each, cap, cap]
    taken = n_pages - 1 - torch.arange(2 * width, dtype=torch.int32, device="cuda")  # from the top of the stack
    assert torch.equal(pages.table[:2].view(-1), taken) and int(pages.table[2, 0]) == 0
    step = 2 ** 26
    for at in range(0, cap, step):
        i = torch.arange(at, at + step, dtype=torch.int32, device="cuda")
        assert torch.equal(rows.pos[at:at + step], i % each)
        assert torch.equal(rows.slot[at:at + step], taken[(i // P).long()] * P + i % P)
    ctx.close()


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [(1, 1), (300, 150)])
def test_pools_beyond_4_gib(t, counts):
    """Rows into pages, and attention over them, of a pool whose tensors have more than 2^32 bytes each."""
    say("a pool beyond 4 GiB", t, counts)
    H, Hkv, dh, P, lengths = 8, 2, 128, 64, (300, 150)
    n_pages = 2 ** 32 // (Hkv * P * dh * TD[t].itemsize) + 40
    g, ctx = W.philox(15, t), context(t, H, Hkv, dh, 512)
    k, v = (torch.empty(n_pages, Hkv, P, dh, dtype=TD[t], device="cuda") for _ in range(2))
    table = np.concatenate([n_pages - 1 - g.permutation(7), [3, n_pages // 2 + 1, 0]])[:10].reshape(2, 5)
    pages = Bd.Pages(k, v, ints(table))
    pos = np.concatenate([np.arange(n) for n in lengths])
    slot = np.concatenate([table[r, np.arange(n) // P] * P + np.arange(n) % P for r, n in enumerate(lengths)])
    qkv = dev(g.standard_normal((450, (H + 2 * Hkv) * dh)), t)
    q = torch.zeros(450, H, dh, dtype=TD[t], device="cuda")
    ctx.head_norm_rope_paged(qkv, None, None, Bd.PageRows(ints([0, 300, 450]), ints(pos), ints(slot)), pages, q)
    x = host(qkv).reshape(450, H + 2 * Hkv, dh)
    y, size = heads(x[:, H:H + Hkv], None, pos[None].astype(float), np.zeros(dh // 2, int))
    page, place = torch.from_numpy(slot // P).cuda(), torch.from_numpy(slot % P).cuda()
    within(k[page, :, place], y, heads_tol(y, size, t), "k")
    assert np.array_equal(host(v[page, :, place]), x[:, H + Hkv:])
    take = np.concatenate([np.arange(300 - counts[0], 300), np.arange(450 - counts[1], 450)])
    rows = Bd.PageRows(ints([0, counts[0], sum(counts)]), ints(pos[take]), ints(slot[take]))
    qs, out = q[torch.from_numpy(take).cuda()], torch.zeros(len(take), H * dh, dtype=TD[t], device="cuda")
    ctx.paged_attention(qs, pages, rows, ints(lengths), out, Bd.Scores(block=1))
    stored = host(k[page, :, place])
    for r, (lo, n) in enumerate(((0, 300), (300, 150))):
        rr = slice(0, counts[0]) if r == 0 else slice(counts[0], None)
        want, tol = attend(host(qs)[rr], stored[lo:lo + n], x[lo:lo + n, H + Hkv:], pos[take][rr], t, block=1)
        within(out[rr], want, tol, "request %d" % r)
    assert ctx.poll_status() == 0
    ctx.close()


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("m", [3, 300])
def test_sequences_beyond_4_gib(t, m):
    """A sequence of [B, L] caches whose keys lie more than 2^32 bytes apart: rows at its end, in a document of the last tokens."""
    say("a sequence beyond 4 GiB", t, m)
    H, Hkv, dh = 32, 32, 64
    L = 2 ** 32 // (Hkv * dh * TD[t].itemsize) + 777
    g = W.philox(16, t)
    ctx = Bd.Context(Bd.LayerCfg(256, H, Hkv, dh, 256, 1, L, 512, Bd.F32 if t == "f32" else Bd.BF16, 1e-5, 1e4))
    k, v = (torch.zeros(1, L, Hkv, dh, dtype=TD[t], device="cuda") for _ in range(2))
    last = 500
    for x in (k, v):
        x[0, L - last:] = dev(g.standard_normal((last, Hkv, dh)), t)
    doc = torch.zeros(1, L, dtype=torch.int32, device="cuda")
    doc[0, L - last + 40:] = 9
    idx = np.arange(L - m, L)
    q, out = dev(g.standard_normal((m, H, dh)), t), torch.zeros(m, H * dh, dtype=TD[t], device="cuda")
    ctx.partial_attention_masked(q, k, v, Bd.IndexList(ints(idx), ints([0, m])), 1, L, out, Bd.Scores(block=1, doc=doc))
    want, tol = attend(host(q), host(k[0, L - last + 40:]), host(v[0, L - last + 40:]), idx - (L - last + 40), t, block=1)
    within(out, want, tol, "rows")
    ctx.close()
