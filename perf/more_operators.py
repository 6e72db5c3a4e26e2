"""Operators of requests served from a paged key/value cache, and attention rows with masked and reshaped scores, in plain
form and through the library.

  plan    lengths of the requests of a step: pages given and taken back, the page table, every new row's position and slot
  rope    raw q|k|v rows: RMSNorm of every query and key head, rotary embedding with positions on one or several axes, q out,
          keys and values into the rows' slots of the pages
  paged   attention of the requests' new rows over their pages
  masked  exact attention rows of listed queries over a [B, L] cache
  Both attentions: scores capped by a tanh, a bias by the distance, causal order of blocks, prefixes; masked: documents too.

Inputs are random: projections N(0, 1) with some channels of the keys larger than others, gains near one, pages in the order
in which a pool hands them out after a while.
"""
import math

import torch

own = False

EPS, THETA = 1e-5, 10000.0
# hidden, query heads, key-value heads, head_dim, ffn, type: the layers of this repository's workloads
SHAPES = {
    "llada": (4096, 32, 32, 128, 12288, "bf16"),
    "dream": (3584, 28, 4, 128, 18944, "bf16"),
    "small": (512, 8, 2, 64, 1536, "bf16"),
    "tiny": (256, 4, 4, 64, 768, "f32"),
}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a decoding step of a full batch: one new token a request, a page for one in sixteen of them
        dict(name="plan-64-decode", kind="plan", requests=64, longest=4096, chunk=1, page=16, mixed=False),
        # a step of a busy server: prompts in chunks, blocks computed again, requests that end and that fall back
        dict(name="plan-1500-mixed", kind="plan", requests=1500, longest=32768, chunk=512, page=64, mixed=True),
        # one decoding step of a small batch in fp32: what is left of a call when there is next to nothing to do
        dict(name="rope-tiny-f32-8", kind="rope", shape="tiny", rows=8, page=16, axes=1, far=100000),
        # an image's rows in a grouped layer: time, height, width; projections wider than q|k|v; a few rows that got no page
        dict(name="rope-gqa-1277-3axes", kind="rope", shape="dream", rows=1277, page=32, axes=3, far=2000, pad=64, skipped=True),
        # a prompt chunk of a large batch, pairs of columns dealt to the axes in turn
        dict(name="rope-8192-3axes", kind="rope", shape="llada", rows=8192, page=64, axes=3, far=30000, turns=True),
        # one token of one request
        dict(name="paged-b1-decode-4k", kind="paged", shape="llada", requests=1, new=1, longest=4096, page=16, block=1),
        # one token in each of 32 requests of many lengths, grouped heads: the cache is read once, nothing else counts
        dict(name="paged-gqa-b32-decode", kind="paged", shape="dream", requests=32, new=1, longest=32768, page=64, block=1, ragged=True),
        # blocks of 32 tokens that see each other and what came before, scores capped
        dict(name="paged-b16-block32-cap", kind="paged", shape="llada", requests=16, new=32, longest=1280, page=32, block=32, cap=30.0, ragged=True),
        # a long prompt in chunks, causal, grouped heads
        dict(name="paged-gqa-b4-chunk2048", kind="paged", shape="dream", requests=4, new=2048, longest=8192, page=64, block=1, ragged=True),
        # the serving batch of the benchmark, a tenth of its rows, prompts that all rows see and a response in causal blocks, bias by distance
        dict(name="masked-b16-10pct-prefix", kind="masked", shape="llada", batch=16, seq=1280, frac=0.10, block=64, prefix=True, bias=True),
        # documents packed into sequences, every row, both directions
        dict(name="masked-gqa-b4-docs-4096", kind="masked", shape="dream", batch=4, seq=4096, frac=1.0, docs=9),
        # a quarter of the rows of two sequences with capped scores, heads of 64, sequences of two lengths
        dict(name="masked-small-b2-cap", kind="masked", shape="small", batch=2, seq=1001, frac=0.25, cap=20.0, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "rope", "paged", "paged", "paged", "masked", "masked"])
    page = rng.choice([16, 32, 64, 128])
    if kind == "plan":
        return dict(kind=kind, requests=_log_int(rng, 1, 1500), longest=_log_int(rng, 64, 32768), chunk=_log_int(rng, 1, 512), page=page,
                    mixed=rng.random() < 0.7)
    c = dict(kind=kind, shape=rng.choice(["llada", "llada", "dream", "dream", "small", "tiny"]))
    if kind == "rope":
        c.update(rows=_log_int(rng, 1, 8192), page=page, axes=rng.choice([1, 2, 3]), far=_log_int(rng, 100, 1000000), pad=rng.choice([0, 0, 64, 8]),
                 turns=rng.random() < 0.5, skipped=rng.random() < 0.3)
        return c
    c.update(block=rng.choice([0, 1, 1, 16, 32, 100]), prefix=rng.random() < 0.3, bias=rng.random() < 0.3, ragged=rng.random() < 0.7)
    if rng.random() < 0.4:
        c["cap"] = rng.choice([10.0, 30.0, 50.0])
    if kind == "paged":
        c.update(page=page, requests=_log_int(rng, 1, 32))
        if rng.random() < 0.5:  # one token a request, lengths up to the longest
            c.update(new=1, longest=_log_int(rng, 16, 32768))
        else:
            c.update(new=_log_int(rng, 2, 2048))
            c.update(longest=_log_int(rng, c["new"], max(c["new"], 8192)))
        n, m, length = c["requests"], c["new"], c["longest"]
    else:
        c.update(batch=_log_int(rng, 1, 16), seq=_log_int(rng, 33, 4096), frac=1.0 if rng.random() < 0.3 else round(math.exp(rng.uniform(math.log(0.01), 0.0)), 4))
        if rng.random() < 0.4:
            c["docs"] = rng.randint(2, 12)
        n, length = c["batch"], c["seq"]
        m = max(1, round(c["frac"] * length))
    _, H, Hkv, dh, _, _ = SHAPES[c["shape"]]
    most = 4 * 2048 * 6000 * 28 // (4 if c["shape"] == "tiny" else 1)  # (request, head, row, key) quadruples of the largest listed case, fewer in fp32
    keys = 32 * 20000 * 4 * 128
    fit = min(1.0, most / (n * H * m * length), keys / (n * Hkv * length * dh))
    c["requests" if kind == "paged" else "batch"] = max(1, int(n * fit))
    if n * fit < 1.0:
        if kind == "paged":
            c["longest"] = max(c["new"], int(length * n * fit))
        else:
            c["frac"] = round(c["frac"] * n * fit, 5)
    return c


# ---- inputs -------------------------------------------------------------------------------------------

def _lengths(case):
    """Keys of every sequence or request (of many lengths: between a third of the longest and all of it)."""
    B, L = (case["requests"], case["longest"]) if case["kind"] == "paged" else (case["batch"], case["seq"])
    if not case.get("ragged"):
        return [L] * B
    return [max(1, round(L * (1.0 - 0.67 * ((b * 0.7548776662) % 1.0)))) for b in range(B)]


def _counts(case):
    """Rows of every sequence: of a list one to all of its tokens, of a request its new tokens (of many lengths: half to all of `new`)."""
    out = []
    for b, n in enumerate(_lengths(case)):
        if case["kind"] == "paged":
            out.append(min(n, max(1, round(case["new"] * (1.0 - 0.5 * ((b * 0.6180339887) % 1.0 if case.get("ragged") else 0.0))))))
        else:
            r = 0.5 + ((b * 0.6180339887) % 1.0) if case["batch"] > 1 else 1.0
            out.append(n if case["frac"] >= 1.0 else min(n, max(1, round(case["frac"] * n * r))))
    return out


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def _channels(dh, gen):
    return torch.exp(0.5 * torch.randn(dh, device="cuda", generator=gen))


def _offsets(counts):
    off = [0]
    for n in counts:
        off.append(off[-1] + n)
    return off


def _prepare_plan(case, seed):
    """Requests of random lengths that hold their pages in random order, and a pool with the rest and some room."""
    R, P, gen = case["requests"], case["page"], torch.Generator().manual_seed(seed)
    rnd = lambda lo, hi: torch.randint(lo, hi + 1, (R,), generator=gen)  # noqa: E731
    now = rnd(0, case["longest"])
    step = rnd(1, case["chunk"]) if case["mixed"] else torch.ones(R, dtype=torch.int64)
    then = (now + step).clamp_max(case["longest"])
    rows = then - now
    if case["mixed"]:
        what = rnd(0, 9)
        rows = torch.where(what == 0, step.clamp_max(now), rows)  # its last block again
        then = torch.where(what == 0, now, then)
        then = torch.where(what == 1, torch.zeros_like(then), then)  # has ended
        then = torch.where(what == 2, (now - step).clamp_min(0), then)  # falls back
        rows = torch.where((what == 1) | (what == 2), torch.zeros_like(rows), rows).clamp_min(0)
    held, need = (now + P - 1) // P, (then + P - 1) // P
    width = (case["longest"] + P - 1) // P
    n_pages = math.ceil(R * (width + 1) * min(1.0, 0.5 + 1.5 / math.sqrt(R))) + 8  # (half of the longest on average, and five deviations)
    pages = torch.randperm(n_pages, generator=gen)
    table = torch.zeros(R, width, dtype=torch.int64)
    mask = torch.arange(width) < held[:, None]
    given = int(held.sum())
    table[mask] = pages[:given]
    free = torch.zeros(n_pages, dtype=torch.int64)
    free[:n_pages - given] = pages[given:]
    c = lambda t: t.to(torch.int32).cuda()  # noqa: E731
    total = R * case["chunk"]
    s = dict(case=dict(case), page=P, n_pages=n_pages, table=c(table), now=c(now), then=c(then), rows=c(rows), free=c(free), n_free=_ints([n_pages - given]),
             len_out=_ints([0] * R), n_free_out=_ints([0]), offsets=_ints([0] * (R + 1)), pos=_ints([0] * total), slot=_ints([0] * total))
    if own:
        from paper_2603_08026_amd import binding
        # (a plan needs no scratch memory and sees nothing of the pages' contents: the smallest layer's)
        s["handle"] = binding.Context(binding.LayerCfg(256, 4, 1, 64, 256, 1, 16, 0, binding.BF16, EPS, THETA))
        k, v = (torch.empty(n_pages, 1, P, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        s["pages"] = binding.Pages(k, v, s["table"])
        s["out"] = binding.PageRows(s["offsets"], s["pos"], s["slot"])
    return s


def _axes(case, dh):
    """The axis of each of the dh / 2 pairs of columns."""
    half, n = dh // 2, case["axes"]
    if case.get("turns"):
        return [p % n for p in range(half)]
    first = half if n == 1 else half // 2 if n == 2 else half // 4  # (time takes fewer than height and width)
    rest = (half - first) // max(n - 1, 1)
    return [0] * first + [a for a in range(1, n) for _ in range(rest)]


def _prepare_rope(case, seed):
    _, H, Hkv, dh, _, t = SHAPES[case["shape"]]
    td, n, P, A = TYPES[t], case["rows"], case["page"], case["axes"]
    gen, host = torch.Generator(device="cuda").manual_seed(seed), torch.Generator().manual_seed(seed)
    width = (H + 2 * Hkv) * dh
    buf = torch.empty(n, width + case.get("pad", 0), dtype=td, device="cuda").normal_(0.0, 1.0, generator=gen)
    s = dict(case=dict(case), dims=(H, Hkv, dh), td=td, page=P, qkv=buf[:, :width])  # (a view of a wider projection where there is a pad)
    s["qkv"][:, H * dh:(H + Hkv) * dh] *= _channels(dh, gen).to(td).repeat(Hkv)
    s["g_q"], s["g_k"] = ((1.0 + 0.1 * torch.randn(dh, device="cuda", generator=gen)).to(td) for _ in range(2))
    n_pages = (n + P - 1) // P + 4
    s["k"], s["v"] = (torch.empty(n_pages, Hkv, P, dh, dtype=td, device="cuda").normal_(0.0, 1.0, generator=gen) for _ in range(2))
    # a run of tokens through pages in random order, from the middle of one
    at = torch.arange(n) + int(torch.randint(0, P, (1,), generator=host))
    slot = torch.randperm(n_pages, generator=host)[at // P] * P + at % P
    if case.get("skipped"):
        slot[torch.rand(n, generator=host) < 0.05] = -1
    start = int(torch.randint(0, case["far"] + 1, (1,), generator=host))
    pos = start + torch.arange(n)
    if A == 1:
        axis_pos = pos[None]
    else:  # frames of an image, or of a few, of 24 x 36 patches
        frame = torch.arange(n) // 864
        axis_pos = torch.stack([start + frame, start + torch.arange(n) % 864 // 36, start + torch.arange(n) % 36])[:A]
    s["pos"], s["slot"], s["axis_pos"] = (x.to(torch.int32).cuda() for x in (pos, slot, axis_pos))
    s["axes"] = _axes(case, dh)
    s["axis"] = _ints(s["axes"])
    s["offsets"] = _ints([0, n])
    s["q_out"] = torch.zeros(n, H, dh, dtype=td, device="cuda")
    return s


def _keys_and_values(n, Hkv, P, dh, td, gen):
    ch = _channels(dh, gen)
    k = torch.empty(n, Hkv, P, dh, dtype=td, device="cuda").normal_(0.0, 1.0, generator=gen)
    k *= (ch / ch.square().mean().sqrt()).to(td)
    return k, torch.empty(n, Hkv, P, dh, dtype=td, device="cuda").normal_(0.0, 1.0, generator=gen)


def _prepare_scores(case, s, seed, lengths, H):
    """What reshapes or masks the scores."""
    s["cap"], s["block"] = case.get("cap", 0.0), case.get("block", 0)
    s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)]).cuda() if case.get("bias") else None
    s["prefix"] = _ints([int(n * (0.2 + 0.5 * ((b * 0.5698402910 + seed * 0.618) % 1.0))) for b, n in enumerate(lengths)]) if case.get("prefix") else None


def _prepare_paged(case, seed):
    _, H, Hkv, dh, _, t = SHAPES[case["shape"]]
    td, P, R = TYPES[t], case["page"], case["requests"]
    gen, host = torch.Generator(device="cuda").manual_seed(seed), torch.Generator().manual_seed(seed)
    lengths, counts = _lengths(case), _counts(case)
    held = [(n + P - 1) // P for n in lengths]
    width, n_pages = (case["longest"] + P - 1) // P, sum(held) + 4
    pages, off_p = torch.randperm(n_pages, generator=host), _offsets(held)
    table = torch.zeros(R, width, dtype=torch.int64)
    for r in range(R):
        table[r, :held[r]] = pages[off_p[r]:off_p[r + 1]]
    off = _offsets(counts)
    s = dict(case=dict(case), dims=(H, Hkv, dh), td=td, page=P, table=table.to(torch.int32).cuda(), offsets=_ints(off), most=max(counts), len=_ints(lengths))
    s["pos"] = torch.cat([torch.arange(n - m, n) for n, m in zip(lengths, counts)]).to(torch.int32).cuda()
    s["k"], s["v"] = _keys_and_values(n_pages, Hkv, P, dh, td, gen)
    s["q"] = (1.5 * torch.randn(off[-1], H, dh, device="cuda", generator=gen)).to(td)
    s["out"] = torch.zeros(off[-1], H * dh, dtype=td, device="cuda")
    s["doc"] = None
    _prepare_scores(case, s, seed, lengths, H)
    return s


def _prepare_masked(case, seed):
    _, H, Hkv, dh, _, t = SHAPES[case["shape"]]
    td, B, L = TYPES[t], case["batch"], case["seq"]
    gen, host = torch.Generator(device="cuda").manual_seed(seed), torch.Generator().manual_seed(seed)
    lengths, counts = _lengths(case), _counts(case)
    off = _offsets(counts)
    idx = torch.cat([torch.sort(torch.randperm(n, generator=host)[:m])[0] + b * L for b, (n, m) in enumerate(zip(lengths, counts))])
    s = dict(case=dict(case), dims=(H, Hkv, dh), td=td, offsets=_ints(off), idx=idx.to(torch.int32).cuda(), most=max(counts))
    s["len"] = _ints(lengths) if case.get("ragged") else None
    k, v = _keys_and_values(B, Hkv, L, dh, td, gen)
    s["k"], s["v"] = (x.transpose(1, 2).contiguous() for x in (k, v))
    s["q"] = (1.5 * torch.randn(off[-1], H, dh, device="cuda", generator=gen)).to(td)
    s["out"] = torch.zeros(off[-1], H * dh, dtype=td, device="cuda")
    s["doc"] = None
    if case.get("docs"):  # documents of many lengths, and padding behind the last (no document: -1)
        ends = torch.sort(torch.randint(1, L + 1, (B, case["docs"]), generator=host), -1)[0]
        ends[:, -1] = torch.tensor([max(1, n - L // 50) for n in lengths])
        doc = (torch.arange(L)[None, :, None] >= ends[:, None]).sum(-1)
        doc[torch.arange(L)[None] >= ends.amax(-1, keepdim=True)] = -1
        s["doc"] = doc.to(torch.int32).cuda()
    _prepare_scores(case, s, seed, lengths, H)
    return s


def prepare(case, seed):
    s = {"plan": _prepare_plan, "rope": _prepare_rope, "paged": _prepare_paged, "masked": _prepare_masked}[case["kind"]](case, seed)
    return _with_handle(s, case) if own and case["kind"] != "plan" else s


def _with_handle(s, case):
    """What a program keeps for the library's calls: a context (scratch memory) and descriptions of its tensors."""
    from paper_2603_08026_amd import binding
    hidden, H, Hkv, dh, ffn, t = SHAPES[case["shape"]]
    B, L = (case["batch"], case["seq"]) if case["kind"] == "masked" else (1, 1280)
    rows = s["q" if "q" in s else "qkv"].shape[0]
    B = max(B, (rows + L - 1) // L)
    s["handle"] = binding.Context(binding.LayerCfg(hidden, H, Hkv, dh, ffn, B, L, rows, binding.F32 if t == "f32" else binding.BF16, EPS, THETA))
    if case["kind"] == "masked":
        s["rows"] = binding.IndexList(s["idx"], s["offsets"])
    else:
        if "table" not in s:
            s["table"] = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
        if "slot" not in s:
            s["slot"] = torch.zeros_like(s["pos"])
        s["pages"] = binding.Pages(s["k"], s["v"], s["table"])
        s["rows"] = binding.PageRows(s["offsets"], s["pos"], s["slot"])
    if "cap" in s:
        s["scores"] = binding.Scores(cap=s["cap"], block=s["block"], prefix=s["prefix"], slopes=s["slopes"], doc=s["doc"])
    return s


# ---- plain forms --------------------------------------------------------------------------------------

def _plain_plan(s):
    P, table, free = s["page"], s["table"], s["free"]
    now, then, want = s["now"].long(), s["then"].long(), s["rows"].long()
    held, need = (now + P - 1) // P, (then + P - 1) // P
    gain, loss = (need - held).clamp_min(0), (held - need).clamp_min(0)
    back, ends = loss.sum(), gain.cumsum(0)
    have = s["n_free"].long() + back
    served = (gain == 0) | (ends <= have)
    taken = (gain * served).sum()
    entry = torch.arange(table.shape[1], device="cuda")
    returned = table[(entry >= need[:, None]) & (entry < held[:, None])]  # in the order of requests and entries
    stack = torch.cat([free[:s["n_free"]], returned.flip(0)])  # what comes back lies on top, the first of it topmost
    grown = (entry >= held[:, None]) & (entry < need[:, None]) & served[:, None]
    table[grown] = stack.flip(0)[:taken]
    left = returned[taken:]
    free[s["n_free"]:s["n_free"] + left.numel()] = left
    s["n_free_out"].copy_(have - taken)
    s["len_out"].copy_(torch.where(served, then, now))
    s["offsets"][1:] = want.cumsum(0)
    req = torch.repeat_interleave(torch.arange(want.numel(), device="cuda"), want)
    pos = then[req] - want[req] + torch.arange(req.numel(), device="cuda") - s["offsets"][req]
    slot = table[req, pos // P].long() * P + pos % P
    s["pos"][:req.numel()] = pos.int()
    s["slot"][:req.numel()] = torch.where(served[req], slot, -1).int()
    return [table, free, s["n_free_out"], s["len_out"], s["offsets"], s["pos"], s["slot"]]


def _plain_rope(s):
    H, Hkv, dh = s["dims"]
    half = dh // 2
    x = s["qkv"].float().reshape(-1, H + 2 * Hkv, dh)
    a = s["axis_pos"][s["axis"].long()].double().t() * THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    co, si = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]
    y = x[:, :H + Hkv]
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
    y = y * torch.cat([s["g_q"].float().expand(H, dh), s["g_k"].float().expand(Hkv, dh)])
    y1, y2 = y[..., :half], y[..., half:]
    y = torch.cat([y1 * co - y2 * si, y2 * co + y1 * si], -1)
    s["q_out"].copy_(y[:, :H])
    some = s["slot"] >= 0
    slot = s["slot"][some].long()
    s["k"][slot // s["page"], :, slot % s["page"]] = y[some, H:].to(s["td"])
    s["v"][slot // s["page"], :, slot % s["page"]] = x[some, H + Hkv:].to(s["td"])
    return [s["q_out"], s["k"], s["v"]]


def _plain_attend(s, k, v, seq, pos):
    """Rows of attention over k, v [B, Hkv, N, dh]: row j is at position pos[j] of sequence seq[j]."""
    H, Hkv, dh = s["dims"]
    g, most, (B, _, N, _) = H // Hkv, s["most"], k.shape
    at = torch.arange(seq.numel(), device="cuda") - s["offsets"].long()[seq]
    q = torch.zeros(B, most, H, dh, device="cuda")
    q[seq, at] = s["q"].float()
    i = torch.zeros(B, most, dtype=torch.int64, device="cuda")
    i[seq, at] = pos
    q = q.view(B, most, Hkv, g, dh).permute(0, 2, 3, 1, 4).reshape(B, Hkv, g * most, dh)
    p = torch.matmul(q, k.transpose(-1, -2).contiguous()).view(B, Hkv, g, most, N)
    p *= 1.0 / math.sqrt(dh)
    if s["cap"] > 0:
        p = p.div_(s["cap"]).tanh_().mul_(s["cap"])
    j = torch.arange(N, device="cuda")
    if s["slopes"] is not None:
        p -= s["slopes"].view(1, Hkv, g, 1, 1) * (i[..., None] - j).abs().float()[:, None, None]
    n = torch.full((B,), N, device="cuda") if s["len"] is None else s["len"].long()
    upto = n[:, None].expand(B, most)
    if s["block"] > 0:
        upto = torch.minimum(upto, (i // s["block"] + 1) * s["block"])
        if s["prefix"] is not None:
            upto = torch.maximum(upto, torch.minimum(s["prefix"].long(), n)[:, None])
    hidden = j >= upto[..., None]
    if s["doc"] is not None:
        mine = torch.gather(s["doc"], 1, i)[..., None]
        hidden |= (s["doc"][:, None] != mine) | (mine < 0)
    p.masked_fill_(hidden[:, None, None], -math.inf)
    p = torch.exp_(p - p.amax(-1, keepdim=True).clamp_min(-3e38))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, g * most, N), v).view(B, Hkv, g, most, dh) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, most, H * dh)
    return o[seq, at].to(s["td"])


def _sequence_of_rows(s):
    off = s["offsets"].long()
    return torch.repeat_interleave(torch.arange(off.numel() - 1, device="cuda"), off[1:] - off[:-1])


def _plain_paged(s):
    H, Hkv, dh = s["dims"]
    R, width = s["table"].shape
    k, v = (x[s["table"].long()].float().transpose(1, 2).reshape(R, Hkv, width * s["page"], dh) for x in (s["k"], s["v"]))
    return _plain_attend(s, k, v, _sequence_of_rows(s), s["pos"].long())


def _plain_masked(s):
    L = s["k"].shape[1]
    k, v = (x.transpose(1, 2).float().contiguous() for x in (s["k"], s["v"]))
    idx = s["idx"].long()
    return _plain_attend(s, k, v, idx // L, idx % L)


def run(s):
    if own:
        return _own(s)
    return {"plan": _plain_plan, "rope": _plain_rope, "paged": _plain_paged, "masked": _plain_masked}[s["case"]["kind"]](s)


def _own(s):
    h, kind = s["handle"], s["case"]["kind"]
    if kind == "plan":
        h.page_plan(s["pages"], s["now"], s["then"], s["rows"], s["free"], s["n_free"], s["out"], s["len_out"], s["n_free_out"])
        return [s["table"], s["free"], s["n_free_out"], s["len_out"], s["offsets"], s["pos"], s["slot"]]
    if kind == "rope":
        h.head_norm_rope_paged(s["qkv"], s["g_q"], s["g_k"], s["rows"], s["pages"], s["q_out"], s["axis_pos"], s["axes"])
        return [s["q_out"], s["k"], s["v"]]
    if kind == "paged":
        h.paged_attention(s["q"], s["pages"], s["rows"], s["len"], s["out"], s["scores"])
    else:
        B, L = s["k"].shape[:2]
        h.partial_attention_masked(s["q"], s["k"], s["v"], s["rows"], B, L, s["out"], s["scores"], s["len"])
    return s["out"]


# ---- what a pass cannot do without --------------------------------------------------------------------

def _visible(case):
    """About how many keys the rows of each sequence see, all rows of the sequence together."""
    out = []
    for n, m in zip(_lengths(case), _counts(case)):
        b = case.get("block", 0)
        if b == 0:
            see = m * n
        elif case["kind"] == "paged":  # the last m positions
            see = m * (n - m) + m * (min(m, b) + m) / 2 if m > 1 else n
        else:  # spread over the sequence
            see = m * n * (0.61 if case.get("prefix") else 0.5)
        out.append(see * (2 / (case["docs"] + 1) if case.get("docs") else 1))  # (pieces cut at random)
    return out


def work(case):
    kind = case["kind"]
    if kind == "plan":
        R = case["requests"]
        rows = R * (case["chunk"] / 2 if case["mixed"] else 1)
        return {"bytes": int(16 * R + 8 * rows + 8 * rows / case["page"]), "flops": int(10 * rows)}
    _, H, Hkv, dh, _, t = SHAPES[case["shape"]]
    e = 4 if t == "f32" else 2
    if kind == "rope":
        n = case["rows"]
        return {"bytes": 2 * n * (H + 2 * Hkv) * dh * e + n * (4 + 4 * case["axes"]), "flops": 9 * n * (H + Hkv) * dh}
    keys = 2 * sum(_lengths(case)) * Hkv * dh * e
    return {"bytes": keys + 2 * sum(_counts(case)) * H * dh * e, "flops": int(4 * sum(_visible(case)) * H * dh)}


# ---- the definitions in 64 bits -----------------------------------------------------------------------

def _exact_rope(s):
    H, Hkv, dh = s["dims"]
    x = s["qkv"].reshape(-1, H + 2 * Hkv, dh).double()
    c = torch.arange(dh, device="cuda")
    pair = c % (dh // 2)
    where = torch.stack([s["axis_pos"][a].double() for a in s["axes"]], 1)[:, pair]  # [n, dh]
    angle = where * torch.pow(torch.tensor(THETA, dtype=torch.float64, device="cuda"), -2.0 * pair.double() / dh)
    out = []
    for heads, g in ((x[:, :H], s["g_q"]), (x[:, H:H + Hkv], s["g_k"])):
        y = heads / torch.sqrt((heads * heads).sum(-1, keepdim=True) / dh + EPS) * g.double()
        partner = torch.roll(y, dh // 2, -1) * torch.where(c < dh // 2, -1.0, 1.0)
        out.append(y * torch.cos(angle)[:, None] + partner * torch.sin(angle)[:, None])
    k, v = s["k"].double(), s["v"].double()
    for j, slot in enumerate(s["slot"].tolist()):
        if slot >= 0:
            k[slot // s["page"], :, slot % s["page"]] = out[1][j]
            v[slot // s["page"], :, slot % s["page"]] = x[j, H + Hkv:]
    return [out[0], k, v]


def _exact_attend(s, keys_of, seq_pos):
    H, Hkv, dh = s["dims"]
    g, off, block = H // Hkv, s["offsets"].tolist(), s["block"]
    out = torch.zeros(off[-1], H, dh, dtype=torch.float64, device="cuda")
    for b in range(len(off) - 1):
        lo, hi = off[b], off[b + 1]
        k_all, v_all, n = keys_of(b)
        i, j = seq_pos(lo, hi).view(-1, 1), torch.arange(n, device="cuda").view(1, -1)
        seen = torch.ones(hi - lo, n, dtype=torch.bool, device="cuda")
        if block:
            seen = torch.div(j, block, rounding_mode="floor") <= torch.div(i, block, rounding_mode="floor")
            if s["prefix"] is not None:
                seen = seen | (j < s["prefix"][b])
        if s["doc"] is not None:
            d = s["doc"][b]
            seen = seen & (d[i] == d[:n]) & (d[i] >= 0)
        for h in range(H):
            x = s["q"][lo:hi, h].double() @ k_all[:n, h // g].double().t().contiguous() / math.sqrt(dh)
            if s["cap"] > 0:
                x = s["cap"] * torch.tanh(x / s["cap"])
            if s["slopes"] is not None:
                x = x - s["slopes"][h].double() * (i - j).abs()
            w = torch.softmax(torch.where(seen, x, -math.inf), -1)
            out[lo:hi, h] = torch.where(seen.any(-1, keepdim=True), w, 0.0) @ v_all[:n, h // g].double()
    return out.view(off[-1], H * dh)


def exact(case, seed):
    global own
    if case["kind"] == "plan":
        return None  # whole numbers
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "rope":
        return _exact_rope(s)
    lengths = _lengths(case)
    if case["kind"] == "paged":
        def keys_of(b):
            t, n = s["table"][b].long(), lengths[b]
            return (*(x[t].transpose(1, 2).flatten(0, 1) for x in (s["k"], s["v"])), n)
        return _exact_attend(s, keys_of, lambda lo, hi: s["pos"][lo:hi].long())
    L = case["seq"]
    return _exact_attend(s, lambda b: (s["k"][b], s["v"][b], lengths[b]), lambda lo, hi: s["idx"][lo:hi].long() % L)
