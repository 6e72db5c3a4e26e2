"""Operators on the heads of a row and on a key/value cache held in 8 bits, in plain form and through the library.

  norm    raw q|k|v rows of listed tokens: RMSNorm of every query and key head, rotary embedding, q out, k and v merged
          into the caches
  store   the same into a cache of 8 bit codes with a scale per (token, key-value head), and the written rows read back
  write   finished k and v rows into such a cache, and read back
  attend  exact attention rows of listed queries over such a cache, of sequences padded to one length

Inputs are random: projections N(0, 1) with some channels of the keys larger than others, gains near one, as after a
random-init layer.
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
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def listed():
    return [
        # one tiny fp32 layer, a tenth of 128 tokens: what is left of a call when there is next to nothing to do
        dict(name="norm-tiny-f32", kind="norm", shape="tiny", batch=1, seq=128, frac=0.10),
        # grouped heads, odd request count and length, rows of a wider projection (a row stride of its own)
        dict(name="norm-gqa-b13-7pct", kind="norm", shape="dream", batch=13, seq=1277, frac=0.07, pad=64),
        # a dense warm-up step of the serving batch: every token
        dict(name="norm-b16-all", kind="norm", shape="llada", batch=16, seq=1280, frac=1.0),
        # interactive use: a tenth of one request's tokens
        dict(name="store-b1-10pct-e4m3", kind="store", shape="llada", batch=1, seq=1024, frac=0.10, codes="e4m3"),
        # serving batch, a quarter of the tokens, the other format
        dict(name="store-b16-25pct-int8", kind="store", shape="llada", batch=16, seq=1280, frac=0.25, codes="int8"),
        # a cache of the serving batch, converted whole
        dict(name="write-b16-all-e4m3", kind="write", shape="llada", batch=16, seq=1280, frac=1.0, codes="e4m3"),
        # one token of one request
        dict(name="attend-b1-1row", kind="attend", shape="llada", batch=1, seq=1024, frac=0.0, codes="e4m3"),
        # one token in each of eight long sequences: the cache is read once, nothing else counts
        dict(name="attend-b8-1row-32k", kind="attend", shape="llada", batch=8, seq=32768, frac=0.0, codes="e4m3"),
        # serving batch at the salient share of trained models, sequences of many lengths in one padded batch
        dict(name="attend-b16-2pct-int8", kind="attend", shape="llada", batch=16, seq=1280, frac=0.02, codes="int8", ragged=True),
        # the benchmark's workload
        dict(name="attend-b16-10pct", kind="attend", shape="llada", batch=16, seq=1280, frac=0.10, codes="e4m3"),
        # grouped heads (28 over 4), odd request count and length
        dict(name="attend-gqa-b13-7pct-int8", kind="attend", shape="dream", batch=13, seq=1277, frac=0.07, codes="int8"),
        # long sequences, a quarter of the tokens: the products count, not the cache
        dict(name="attend-b16-25pct-2048", kind="attend", shape="llada", batch=16, seq=2048, frac=0.25, codes="e4m3"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "store", "write", "attend", "attend", "attend", "attend"])
    c = dict(kind=kind, shape=rng.choice(["llada", "llada", "dream", "dream", "small", "tiny"]))
    c["batch"] = _log_int(rng, 1, 16)
    if kind != "norm":
        c["codes"] = rng.choice(["e4m3", "int8"])
    if kind != "attend":
        c["seq"] = _log_int(rng, 16, 1280)
        c["frac"] = 1.0 if rng.random() < 0.25 else round(math.exp(rng.uniform(math.log(0.01), 0.0)), 4)
        if kind != "write":
            c["pad"] = rng.choice([0, 0, 64, 8])
        return c
    c["ragged"] = rng.random() < 0.5
    if rng.random() < 0.35:  # one row a sequence, lengths up to the longest
        c["seq"], c["frac"] = _log_int(rng, 16, 262144 // 8 // (1 if c["batch"] <= 8 else 2)), 0.0
    else:
        c["seq"] = _log_int(rng, 33, 2048)
        c["frac"] = round(math.exp(rng.uniform(math.log(0.01), math.log(0.25))), 4)
    return c


# ---- inputs -------------------------------------------------------------------------------------------

def _lengths(case):
    """Keys of every sequence (a padded batch: between a third of the longest and all of it)."""
    B, L = case["batch"], case["seq"]
    if not case.get("ragged"):
        return [L] * B
    return [max(1, round(L * (1.0 - 0.67 * ((b * 0.7548776662) % 1.0)))) for b in range(B)]


def _counts(case):
    """Listed rows of every sequence: all, one, or 0.5 .. 1.5 times the share of its tokens."""
    out = []
    for b, n in enumerate(_lengths(case)):
        r = 0.5 + ((b * 0.6180339887) % 1.0) if case["batch"] > 1 else 1.0
        out.append(n if case["frac"] >= 1.0 else min(n, max(1, round(case["frac"] * n * r))))
    return out


def _rows(case, seed):
    """Ascending token ids b * L + i and the offsets of the sequences."""
    gen = torch.Generator().manual_seed(seed)
    ids, off = [], [0]
    for b, (n, m) in enumerate(zip(_lengths(case), _counts(case))):
        ids.append(torch.sort(torch.randperm(n, generator=gen)[:m])[0] + b * case["seq"])
        off.append(off[-1] + m)
    return torch.cat(ids).to(torch.int32).cuda(), torch.tensor(off, dtype=torch.int32).cuda()


def _channels(dh, gen):
    return torch.exp(0.5 * torch.randn(dh, device="cuda", generator=gen))


def prepare(case, seed):
    _, H, Hkv, dh, _, t = SHAPES[case["shape"]]
    B, L, kind, td = case["batch"], case["seq"], case["kind"], TYPES[t]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    idx, off = _rows(case, seed)
    n = idx.numel()
    s = dict(case=dict(case), dims=(B, L, H, Hkv, dh), td=td, idx=idx, off=off)
    if kind in ("norm", "store"):
        width = (H + 2 * Hkv) * dh
        buf = torch.empty(n, width + case.get("pad", 0), dtype=td, device="cuda").normal_(0.0, 1.0, generator=gen)
        s["qkv"] = buf[:, :width]  # (a view of a wider projection where there is a pad)
        s["qkv"][:, H * dh:(H + Hkv) * dh] *= _channels(dh, gen).to(td).repeat(Hkv)
        s["g_q"], s["g_k"] = (1.0 + 0.1 * rnd(dh)).to(td), (1.0 + 0.1 * rnd(dh)).to(td)
        s["q_out"] = torch.zeros(n, H, dh, dtype=td, device="cuda")
    if kind == "norm":
        s["k"] = torch.empty(B, L, Hkv, dh, dtype=td, device="cuda").normal_(0.0, 1.0, generator=gen)
        s["v"] = torch.empty(B, L, Hkv, dh, dtype=td, device="cuda").normal_(0.0, 1.0, generator=gen)
        return _with_handle(s)
    codes = CODES[case["codes"]]
    if kind == "attend":
        s["q"] = (1.5 * rnd(n, H, dh)).to(td)
        ch = _channels(dh, gen)
        s["kc"], s["ks"] = _quantise(rnd(B, L, Hkv, dh) * (ch / ch.square().mean().sqrt()), codes)
        s["vc"], s["vs"] = _quantise(rnd(B, L, Hkv, dh), codes)
        s["len"] = torch.tensor(_lengths(case), dtype=torch.int32).cuda() if case.get("ragged") else None
        s["most"] = max(_counts(case))
        s["out"] = torch.zeros(n, H * dh, dtype=td, device="cuda")
    else:
        if kind == "write":
            s["k"] = (rnd(n, Hkv, dh) * _channels(dh, gen)).to(td)
            s["v"] = rnd(n, Hkv, dh).to(td)
        s["kc"], s["vc"] = (torch.zeros(B, L, Hkv, dh, device="cuda").to(codes) for _ in range(2))
        s["ks"], s["vs"] = (torch.zeros(B, Hkv, L, device="cuda") for _ in range(2))
        s["k_back"], s["v_back"] = (torch.zeros(n, Hkv, dh, dtype=td, device="cuda") for _ in range(2))
    return _with_handle(s)


def _with_handle(s):
    """What a program keeps for the library's calls: a context (scratch memory) and descriptions of its tensors."""
    if not own:
        return s
    from paper_2603_08026_amd import binding
    case = s["case"]
    hidden, H, Hkv, dh, ffn, t = SHAPES[case["shape"]]
    s["handle"] = binding.Context(binding.LayerCfg(hidden, H, Hkv, dh, ffn, case["batch"], case["seq"], sum(_counts(case)),
                                                   binding.F32 if t == "f32" else binding.BF16, EPS, THETA))
    s["rows"] = binding.IndexList(s["idx"], s["off"])
    if "kc" in s:
        s["cache"] = binding.QuantCache(s["kc"], s["vc"], s["ks"], s["vs"])
    elif "k" in s:
        none = torch.zeros(8, dtype=s["td"], device="cuda")
        s["cache"], s["none"] = binding.make_cache(s["k"], s["v"], none, none), none
    return s


# ---- plain forms --------------------------------------------------------------------------------------

def _quantise(y, codes):
    """[B, L, Hkv, dh] fp32 -> codes of the same layout and scales [B, Hkv, L]."""
    m = y.abs().amax(-1).clamp_min(2.0 ** -100)
    if codes == torch.int8:
        c, scale = torch.round(y * (127.0 / m)[..., None]).to(torch.int8), m / 127.0
    else:
        f, e = torch.frexp(m)  # m = f 2^e, 0.5 <= f < 1;  448 = 0.875 * 2^9
        scale = torch.ldexp(torch.ones_like(m), (e - 9 + (f > 0.875).int()).clamp_min(-100))
        c = (y / scale[..., None]).to(torch.float8_e4m3fn)
    return c, scale.transpose(-1, -2).contiguous()


def _normed(x, g):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * g.float()


def _rotated(x, pos):
    half = x.shape[-1] // 2
    a = pos.double()[:, None] * THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    co, si = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]
    x1, x2 = x[..., :half], x[..., half:]
    return torch.cat((x1 * co - x2 * si, x2 * co + x1 * si), -1)


def _plain_heads(s):
    B, L, H, Hkv, dh = s["dims"]
    x = s["qkv"].float().reshape(-1, H + 2 * Hkv, dh)
    pos = s["idx"] % L
    q = _rotated(_normed(x[:, :H], s["g_q"]), pos)
    k = _rotated(_normed(x[:, H:H + Hkv], s["g_k"]), pos)
    return q, k, x[:, H + Hkv:]


def _plain_store(s, k, v):
    B, L, H, Hkv, dh = s["dims"]
    idx = s["idx"].long()
    back = []
    for y, c, sc in ((k, s["kc"], s["ks"]), (v, s["vc"], s["vs"])):
        codes, scale = _quantise(y[None], c.dtype)  # scale [1, Hkv, n]
        c.view(torch.uint8).view(B * L, Hkv, dh)[idx] = codes[0].view(torch.uint8)
        sc[idx // L, :, idx % L] = scale[0].t()
        read = c.view(torch.uint8).view(B * L, Hkv, dh)[idx].view(c.dtype).float()
        back.append((read * sc[idx // L, :, idx % L][..., None]).to(s["td"]))
    return back


def _plain_attend(s):
    B, L, H, Hkv, dh = s["dims"]
    g, most = H // Hkv, s["most"]
    idx = s["idx"].long()
    seq = idx // L
    slot = torch.arange(idx.numel(), device="cuda") - s["off"].long()[seq]
    q = torch.zeros(B, most, H, dh, device="cuda")
    q[seq, slot] = s["q"].float()
    q = q.view(B, most, Hkv, g, dh).permute(0, 2, 1, 3, 4).reshape(B, Hkv, most * g, dh)
    k = s["kc"].float().permute(0, 2, 1, 3) * s["ks"][..., None]
    v = s["vc"].float().permute(0, 2, 1, 3) * s["vs"][..., None]
    p = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(dh))
    if s["len"] is not None:
        p.masked_fill_((torch.arange(L, device="cuda") >= s["len"][:, None])[:, None, None], -math.inf)
    p = torch.exp_(p - p.amax(-1, keepdim=True))
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    o = o.view(B, Hkv, most, g, dh).permute(0, 2, 1, 3, 4).reshape(B, most, H * dh)
    return o[seq, slot].to(s["td"])


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own(s, kind)
    if kind == "attend":
        return _plain_attend(s)
    if kind == "write":
        return _plain_store(s, s["k"].float(), s["v"].float())
    q, k, v = _plain_heads(s)
    if kind == "store":
        return [q.to(s["td"])] + _plain_store(s, k, v)
    B, L, H, Hkv, dh = s["dims"]
    idx = s["idx"].long()
    s["k"].view(B * L, Hkv, dh)[idx] = k.to(s["td"])
    s["v"].view(B * L, Hkv, dh)[idx] = v.to(s["td"])
    return [q.to(s["td"]), s["k"], s["v"]]


def _own(s, kind):
    h, (B, L, H, Hkv, dh) = s["handle"], s["dims"]
    if kind == "attend":
        h.partial_attention_quant(s["q"], s["cache"], s["rows"], B, L, s["out"], s["len"])
        return s["out"]
    if kind == "norm":
        h.head_norm_rope(s["qkv"], s["g_q"], s["g_k"], s["rows"], B, L, s["cache"], s["q_out"])
        return [s["q_out"], s["k"], s["v"]]
    if kind == "store":
        h.head_norm_rope_quant(s["qkv"], s["g_q"], s["g_k"], s["rows"], B, L, s["cache"], s["q_out"])
    else:
        h.quant_write(s["k"], s["v"], s["rows"], B, L, s["cache"])
    h.quant_read(s["cache"], s["rows"], B, L, s["k_back"], s["v_back"])
    return ([s["q_out"]] if kind == "store" else []) + [s["k_back"], s["v_back"]]


# ---- what a pass cannot do without --------------------------------------------------------------------

def work(case):
    _, H, Hkv, dh, _, t = SHAPES[case["shape"]]
    e, counts, kind = (4 if t == "f32" else 2), _counts(case), case["kind"]
    n = sum(counts)
    kv = 2 * n * Hkv
    if kind == "attend":
        keys = sum(_lengths(case)) * 2 * Hkv * (dh + 4)
        return {"bytes": keys + 2 * n * H * dh * e, "flops": sum(4 * m * k * H * dh for m, k in zip(counts, _lengths(case)))}
    if kind == "write":
        return {"bytes": kv * (dh * e + (dh + 4) * 2 + dh * e), "flops": 3 * kv * dh}
    rows = n * (H + 2 * Hkv) * dh * e + n * dh * 4
    if kind == "norm":
        return {"bytes": rows + n * (H + 2 * Hkv) * dh * e, "flops": 9 * n * (H + Hkv) * dh}
    return {"bytes": rows + n * H * dh * e + kv * (dh + 4) * 2 + kv * dh * e, "flops": 9 * n * (H + Hkv) * dh + 3 * kv * dh}


# ---- the definitions in 64 bits -----------------------------------------------------------------------

def _exact_head(x, g, pos, dh):
    x = x.double()
    x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / dh + EPS) * g.double()
    i = torch.arange(dh, device="cuda")
    ang = pos.double().view(-1, 1, 1) * torch.pow(torch.tensor(THETA, dtype=torch.float64, device="cuda"), -2.0 * (i % (dh // 2)).double() / dh)
    partner = torch.roll(x, dh // 2, -1) * torch.where(i < dh // 2, -1.0, 1.0)
    return x * torch.cos(ang) + partner * torch.sin(ang)


def _exact_round_trip(y, codes):
    y = y.double()
    m = y.abs().max(-1, keepdim=True)[0].clamp(min=2.0 ** -100)
    if codes == "int8":
        return torch.round(y * (127.0 / m)) * (m / 127.0)
    step = torch.exp2(torch.ceil(torch.log2(m / 448.0)).clamp(min=-100.0))
    z = y / step  # at most 448: four significant bits, and steps of 2^-9 below 2^-6
    ulp = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(z / ulp) * ulp * step


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    B, L, H, Hkv, dh = s["dims"]
    kind, idx = case["kind"], s["idx"].long()
    if kind == "attend":
        out = torch.empty(idx.numel(), H, dh, dtype=torch.float64, device="cuda")
        off = s["off"].tolist()
        for b, n in enumerate(_lengths(case)):
            lo, hi = off[b], off[b + 1]
            for h in range(Hkv):
                hs = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
                k = s["kc"][b, :n, h].double() * s["ks"][b, h, :n, None].double()
                v = s["vc"][b, :n, h].double() * s["vs"][b, h, :n, None].double()
                q = s["q"][lo:hi, hs].double().reshape(-1, dh)
                out[lo:hi, hs] = (torch.softmax((q @ k.t().contiguous()) / math.sqrt(dh), -1) @ v).view(hi - lo, -1, dh)
        return out.view(-1, H * dh)
    if kind == "write":
        return [_exact_round_trip(s["k"], case["codes"]), _exact_round_trip(s["v"], case["codes"])]
    x, pos = s["qkv"].reshape(-1, H + 2 * Hkv, dh), idx - idx // L * L
    q = _exact_head(x[:, :H], s["g_q"], pos, dh)
    k = _exact_head(x[:, H:H + Hkv], s["g_k"], pos, dh)
    v = x[:, H + Hkv:].double()
    if kind == "store":
        return [q, _exact_round_trip(k, case["codes"]), _exact_round_trip(v, case["codes"])]
    kc, vc = s["k"].double(), s["v"].double()
    kc.view(B * L, Hkv, dh)[idx] = k
    vc.view(B * L, Hkv, dh)[idx] = v
    return [q, kc, vc]
