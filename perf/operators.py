"""Timed cases: the operators around the GEMMs of a decoder layer that serves from a paged key/value cache.

  norm   the residual step between two blocks: r = x + scale gate * N(h), y = N(r), with the norm
         after a block, its gate and the norm before the next block in one pass
  rope   rotary positions of the new tokens' queries and keys, straight from the QKV projection's
         rows; the keys and values go to their pages of the cache
  attn   attention of the new tokens (one a sequence when decoding, a chunk of them before that)
         over everything that the cache holds of their sequences

``prepare`` draws a case's inputs on the GPU, ``run`` is one pass: the plain form in 32 bits, or
(``own``) the calls that a user makes.  ``exact`` is the definition in 64 bits.  The lengths of a
ragged batch follow from the case alone (``_lengths``), so that ``work`` can count them.
"""
import math

import torch

own = False
_ctx = None

PAGE = 64


def listed():
    return [
        # between two blocks of a decoder that answers 4 requests: one launch, latency
        {"name": "norm_b4", "kind": "norm", "R": 4, "C": 2048, "post": "none", "pre": "rms", "gate": "none", "res": "bf16"},
        # a chunk of prompt tokens, norms before and after the block, 32-bit residual stream
        {"name": "norm_8192", "kind": "norm", "R": 8192, "C": 4096, "post": "rms", "pre": "rms", "gate": "none", "res": "f32"},
        # ViT-B/16's tokens at batch 32 with a gate per image and layer norm
        {"name": "norm_vit", "kind": "norm", "R": 6304, "C": 768, "post": "none", "pre": "layer", "gate": "group", "res": "bf16"},
        # one new token for each of 64 requests, whole heads, halves rotated
        {"name": "rope_b64", "kind": "rope", "B": 64, "n": 1, "kv_min": 200, "kv_max": 2000, "heads": 32, "kv_heads": 8, "hd": 128,
         "rot": 128, "layout": "half", "scaling": "none"},
        # a long prompt's chunk far into its context: interleaved, half of each head, stretched positions
        {"name": "rope_8k", "kind": "rope", "B": 1, "n": 8191, "kv_min": 32767, "kv_max": 32767, "heads": 32, "kv_heads": 8, "hd": 128,
         "rot": 64, "layout": "interleaved", "scaling": "parts"},
        # a few requests with short contexts on ViT-B/16's heads: latency
        {"name": "attn_decode_short", "kind": "attn", "B": 4, "n": 1, "kv_min": 100, "kv_max": 500, "heads": 12, "kv_heads": 12, "hd": 64,
         "causal": True, "window": 0, "lse": False, "hole": False},
        # one token for each of 64 requests, contexts of very different lengths
        {"name": "attn_decode_b64", "kind": "attn", "B": 64, "n": 1, "kv_min": 500, "kv_max": 16000, "heads": 32, "kv_heads": 8, "hd": 128,
         "causal": True, "window": 0, "lse": False, "hole": False},
        # one request with a very long context: the keys are split over the whole GPU
        {"name": "attn_decode_long", "kind": "attn", "B": 1, "n": 1, "kv_min": 131071, "kv_max": 131071, "heads": 32, "kv_heads": 8,
         "hd": 128, "causal": True, "window": 0, "lse": True, "hole": False},
        # drafted tokens of 16 requests checked at once
        {"name": "attn_draft_b16", "kind": "attn", "B": 16, "n": 5, "kv_min": 1000, "kv_max": 8000, "heads": 32, "kv_heads": 8, "hd": 128,
         "causal": True, "window": 0, "lse": False, "hole": False},
        # chunks of 1 to 512 new tokens beside each other; one request with more of them than cached
        {"name": "attn_chunk_mixed", "kind": "attn", "B": 8, "n": 512, "kv_min": 600, "kv_max": 12000, "heads": 32, "kv_heads": 8, "hd": 128,
         "causal": True, "window": 0, "lse": False, "hole": True},
        # a whole prompt at once
        {"name": "attn_prompt", "kind": "attn", "B": 1, "n": 8191, "kv_min": 8191, "kv_max": 8191, "heads": 32, "kv_heads": 8, "hd": 128,
         "causal": True, "window": 0, "lse": False, "hole": False},
        # sliding window, small heads
        {"name": "attn_window", "kind": "attn", "B": 4, "n": 1000, "kv_min": 1500, "kv_max": 6000, "heads": 16, "kv_heads": 4, "hd": 64,
         "causal": True, "window": 1024, "lse": True, "hole": False},
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(round(v / step)) * step)


def _size(step, v):
    """v, and one step more at the one size that no case takes."""
    return v + step if v == 3072 else v


def _draw(rng):
    kind = rng.choice(["norm", "norm", "rope", "attn", "attn", "attn"])
    if kind == "norm":
        C = _size(8, _log(rng, 64, 8192, 8))
        return {"kind": kind, "R": _size(1, _log(rng, 1, 12000)), "C": C, "post": rng.choice(["none", "rms", "layer"]),
                "pre": rng.choice(["rms", "rms", "layer"]), "gate": rng.choice(["none", "channel", "group"]),
                "res": rng.choice(["bf16", "f32"])}
    group = rng.choice([1, 2, 3, 4, 6, 8])
    kv_heads = rng.choice([1, 2, 4, 8])
    hd = rng.choice([64, 128])
    if group * kv_heads * hd == 3072:
        group += 1
    if kind == "rope":
        n = _log(rng, 1, 8000)
        B = max(1, min(64, _log(rng, 1, max(1, 8000 // n))))
        hi = n + _log(rng, 1, 4000)
        return {"kind": kind, "B": B, "n": n, "kv_min": n, "kv_max": _size(1, hi), "heads": group * kv_heads, "kv_heads": kv_heads,
                "hd": hd, "rot": rng.choice([hd, hd // 2, hd // 4 * 3]), "layout": rng.choice(["half", "interleaved"]),
                "scaling": rng.choice(["none", "linear", "base", "parts"])}
    n = 1 if rng.random() < 0.4 else _log(rng, 2, 4000)
    B = _log(rng, 1, 64) if n == 1 else max(1, min(16, _log(rng, 1, max(1, 6000 // n))))
    hi = n + _log(rng, 1, 100000 if B <= 2 and n <= 8 else 8000)
    lo = max(n, hi // rng.choice([1, 2, 10, 30]))
    return {"kind": kind, "B": B, "n": _size(1, n), "kv_min": _size(1, lo), "kv_max": _size(2, hi) if hi >= lo else _size(1, lo),
            "heads": group * kv_heads, "kv_heads": kv_heads, "hd": hd, "causal": rng.random() < 0.85,
            "window": rng.choice([0, 0, 0, 100, 1000]), "lse": rng.random() < 0.3, "hole": B > 1 and rng.random() < 0.3}


def draw(rng):
    """One more case of the listed ranges, no more work than the largest of its kind."""
    while True:
        c = _draw(rng)
        most = [work(x) for x in listed() if x["kind"] == c["kind"]]
        w = work(c)
        if w["bytes"] > max(m["bytes"] for m in most) or w["flops"] > max(m["flops"] for m in most):
            continue
        # the plain form holds all scores of a padded batch
        if c["kind"] == "attn" and c["B"] * c["heads"] * c["n"] * c["kv_max"] > 32 * 8192 * 8192:
            continue
        return c


# ---------------------------------------------------------------------------
# lengths of a batch: new tokens and cached tokens (the new ones among them) of each sequence
# ---------------------------------------------------------------------------
def _lengths(c):
    B, n, lo, hi = c["B"], c["n"], c["kv_min"], c["kv_max"]
    new, kv = [], []
    for b in range(B):
        u = ((b * 0.6180339887498949) % 1.0) if B > 1 else 1.0
        # lengths spread evenly over their logarithm; chunks from one token to n
        kv.append(max(1, int(round(lo * (hi / lo) ** u))))
        m = n if n <= 8 or b == 0 else max(1, int(round(n ** (((b + 1) * 0.7548776662466927) % 1.0))))
        new.append(min(m, kv[-1]))
    if c.get("hole"):
        kv[-1] = new[-1] // 2  # fewer cached than new: the first of its rows are empty
    return new, kv


def _pairs(n, L, causal, window):
    """Query-key pairs that the mask leaves."""
    total = 0
    for i in range(n):
        p = L - n + i
        top = min(L, p + 1) if causal else L
        low = max(0, p - window + 1) if window else 0
        total += max(0, top - low)
    return total


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _freqs(c):
    """Angular frequencies of the rotated pairs in 64 bits."""
    rot, base = c["rot"], 10000.0
    i = torch.arange(rot // 2, dtype=torch.float64)
    if c["scaling"] == "base":
        base = base * 4.0 ** (rot / (rot - 2.0))
    f = base ** (-2.0 * i / rot)
    if c["scaling"] == "linear":
        f = f / 4.0
    if c["scaling"] == "parts":
        turns = 8192.0 * f / (2.0 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / 4.0)
    return f


def _rope_scale(c):
    return 0.1 * math.log(4.0) + 1.0 if c["scaling"] == "parts" else 1.0


def prepare(case, seed):
    global _ctx
    c, g = case, _gen(seed)
    s = {"case": c}

    def normal(*shape, dtype=torch.bfloat16, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale + shift).to(dtype)

    if c["kind"] == "norm":
        R, C = c["R"], c["C"]
        rt = torch.float32 if c["res"] == "f32" else torch.bfloat16
        # a residual stream grows over the layers and has a few large channels
        chan = torch.exp(0.5 * torch.randn(C, generator=g, device="cuda"))
        s["x"] = (torch.randn(R, C, generator=g, device="cuda") * 3.0 * chan).to(rt)
        s["h"] = normal(R, C)
        for at in ("post", "pre"):
            s[at + "_w"] = normal(C, dtype=torch.float32, scale=0.1, shift=1.0)
            s[at + "_b"] = normal(C, dtype=torch.float32, scale=0.1) if c[at] == "layer" else None
        per = 0
        if c["gate"] == "channel":
            s["gate"] = normal(1, C, dtype=torch.float32, scale=0.3)
        elif c["gate"] == "group":
            per = 197
            s["gate"] = normal((R + per - 1) // per, C, dtype=torch.float32, scale=0.3)
        else:
            s["gate"] = None
        s["per"], s["scale"] = per, 0.7
    else:
        new, kv = _lengths(c)
        B, H, KH, D = c["B"], c["heads"], c["kv_heads"], c["hd"]
        T = sum(new)
        need = [max((max(L, n) + PAGE - 1) // PAGE, 1) for n, L in zip(new, kv)]
        pages = sum(need) + 3
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        width = max(need)
        table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
        cols = torch.arange(width, device="cuda")
        needed = torch.tensor(need, device="cuda")
        first = torch.cumsum(needed, 0) - needed
        live = cols[None] < needed[:, None]
        table[live] = order[(first[:, None] + cols[None])[live]]
        s["table"] = table
        s["q_start"] = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
        s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device="cuda")
        s["max_q"] = max(new)
        if c["kind"] == "rope":
            s["qkv"] = normal(T, (H + 2 * KH) * D)
            s["k"] = torch.zeros(pages, KH, PAGE, D, dtype=torch.bfloat16, device="cuda")
            s["v"] = torch.zeros_like(s["k"])
            s["freq"] = _freqs(c).cuda().to(torch.float32)
        else:
            s["q"] = normal(T, H, D, scale=1.5)
            s["k"] = normal(pages, KH, PAGE, D)
            s["v"] = normal(pages, KH, PAGE, D)
            # what no token has been written to holds anything
            pos = cols[:, None] * PAGE + torch.arange(PAGE, device="cuda")
            unused = torch.ones(pages, PAGE, dtype=torch.bool, device="cuda")
            used = (pos[None] < s["kv_len"][:, None, None]) & live[..., None]
            unused[table[live].long()] = ~used[live]
            s["k"].masked_fill_(unused[:, None, :, None], float("nan"))
            s["v"].masked_fill_(unused[:, None, :, None], float("nan"))
            s["scale"] = 1.0 / math.sqrt(D)
    if own:
        from paper_2511_19457_gb300 import sparoa as sp
        if _ctx is None:
            _ctx = sp.Context(0)
        s["ctx"], s["sp"] = _ctx, sp
        if c["kind"] == "norm":
            s["r"] = torch.empty_like(s["x"])
            s["y"] = torch.empty_like(s["h"])
            for at in ("post", "pre"):
                s[at] = sp.norm(c[at], weight=s[at + "_w"], bias=s[at + "_b"], eps=1e-6)
        else:
            s["cache"] = sp.KVCache(s["k"], s["v"])
            s["batch"] = sp.PagedBatch(s["q_start"], s["kv_len"], s["table"], max_q=s["max_q"])
            if c["kind"] == "rope":
                s["rope"] = sp.Rope(c["rot"], layout=c["layout"], base=10000.0, scaling=c["scaling"], factor=4.0,
                                    context=8192, low=1.0, high=32.0, scale=_rope_scale(c))
                s["q"] = torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda")
            else:
                s["y"] = torch.empty_like(s["q"])
                s["lse"] = torch.empty(T, H, dtype=torch.float32, device="cuda") if c["lse"] else None
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"norm": _own_norm, "rope": _own_rope, "attn": _own_attn}[kind](s)
    return {"norm": _plain_norm, "rope": _plain_rope, "attn": _plain_attn}[kind](s)


def _own_norm(s):
    s["sp"].sparoa_add_norm(s["ctx"], s["x"], s["h"], s["r"], s["y"], post=s["post"], gate=s["gate"],
                            rows_per_gate=s["per"], scale=s["scale"], pre=s["pre"])
    return {"r": s["r"], "y": s["y"]}


def _own_rope(s):
    s["sp"].sparoa_rope_append(s["ctx"], s["qkv"], s["q"], s["cache"], s["batch"], s["rope"])
    return {"q": s["q"], "k": s["k"], "v": s["v"]}


def _own_attn(s):
    c = s["case"]
    s["sp"].sparoa_paged_attention(s["ctx"], s["q"], s["y"], s["cache"], s["batch"], scale=s["scale"], causal=c["causal"],
                                   window=c["window"], lse=s["lse"])
    return {"y": s["y"]} if s["lse"] is None else {"y": s["y"], "lse": s["lse"]}


def _plain_n(v, kind, w, b):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + 1e-6) * w
    return v if b is None else v + b


def _plain_norm(s):
    c = s["case"]
    h = _plain_n(s["h"].float(), c["post"], s["post_w"], s["post_b"]) * s["scale"]
    if s["gate"] is not None:
        gate = s["gate"]
        if s["per"]:
            gate = gate[torch.arange(c["R"], device="cuda") // s["per"]]
        h = h * gate
    r = s["x"].float() + h
    y = _plain_n(r, c["pre"], s["pre_w"], s["pre_b"])
    return {"r": r.to(s["x"].dtype), "y": y.to(torch.bfloat16)}


def _places(s):
    """Sequence and position of every new token."""
    start = s["q_start"].long()
    new = start[1:] - start[:-1]
    t = torch.arange((s["qkv"] if "qkv" in s else s["q"]).shape[0], device="cuda")
    b = torch.searchsorted(start[1:].contiguous(), t, right=True)
    return b, s["kv_len"].long()[b] - new[b] + t - start[b]


def _plain_rope(s):
    c = s["case"]
    H, KH, D, rot = c["heads"], c["kv_heads"], c["hd"], c["rot"]
    b, pos = _places(s)
    x = s["qkv"].view(-1, H + 2 * KH, D)
    ang = pos.float()[:, None] * s["freq"][None]
    cos, sin = torch.cos(ang)[:, None] * _rope_scale(c), torch.sin(ang)[:, None] * _rope_scale(c)
    f = x[:, :H + KH].float()
    out = f.clone()
    if c["layout"] == "half":
        lo, hi = f[..., :rot // 2], f[..., rot // 2:rot]
        out[..., :rot // 2] = lo * cos - hi * sin
        out[..., rot // 2:rot] = hi * cos + lo * sin
    else:
        lo, hi = f[..., :rot:2], f[..., 1:rot:2]
        out[..., :rot:2] = lo * cos - hi * sin
        out[..., 1:rot:2] = hi * cos + lo * sin
    out = out.to(torch.bfloat16)
    page = s["table"].long()[b, pos // PAGE]
    s["k"][page, :, pos % PAGE] = out[:, H:]
    s["v"][page, :, pos % PAGE] = x[:, H + KH:]
    return {"q": out[:, :H].contiguous(), "k": s["k"], "v": s["v"]}


def _plain_attn(s):
    c = s["case"]
    H, KH, D = c["heads"], c["kv_heads"], c["hd"]
    G, B, n = H // KH, c["B"], s["max_q"]
    start = s["q_start"].long()
    new, L = (start[1:] - start[:-1])[:, None], s["kv_len"].long()[:, None]
    i = torch.arange(n, device="cuda")[None]
    at = (start[:-1, None] + i).clamp_max(s["q"].shape[0] - 1)
    q = s["q"][at].float().view(B, n, KH, G, D).permute(0, 2, 3, 1, 4).reshape(B, KH, G * n, D)
    width = s["table"].shape[1]
    table = s["table"].long().clamp_min(0)
    j = torch.arange(width * PAGE, device="cuda")[None]
    there = (j < L)[:, None, :, None]
    k = s["k"][table].permute(0, 2, 1, 3, 4).reshape(B, KH, width * PAGE, D).float()
    k = torch.where(there, k, 0.0)
    pos = L - new + i
    keep = (j < L)[:, None]
    if c["causal"]:
        keep = keep & (j[:, None] <= pos[..., None])
    if c["window"]:
        keep = keep & (j[:, None] > pos[..., None] - c["window"])
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(s["scale"]).view(B, KH, G, n, -1)
    del k
    x.masked_fill_(~keep.expand(B, n, width * PAGE)[:, None, None], float("-inf"))
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)
    p = x.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    v = s["v"][table].permute(0, 2, 1, 3, 4).reshape(B, KH, width * PAGE, D).float()
    v = torch.where(there, v, 0.0)
    o = torch.matmul(p.view(B, KH, G * n, -1), v).view(B, KH, G, n, D)
    o = torch.where(total > 0, o / total, 0.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, n, H, D)
    valid = i < new
    y = o[valid].to(torch.bfloat16)
    if not c["lse"]:
        return {"y": y}
    lse = (m + total.log())[..., 0].permute(0, 3, 1, 2).reshape(B, n, H)
    return {"y": y, "lse": lse[valid]}


# ---------------------------------------------------------------------------
# the work of a pass
# ---------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "norm":
        R, C, res = c["R"], c["C"], 4 if c["res"] == "f32" else 2
        gates = {"none": 0, "channel": 1, "group": (R + 196) // 197}[c["gate"]]
        vecs = sum({"none": 0, "rms": 1, "layer": 2}[c[a]] for a in ("post", "pre")) + gates
        return {"bytes": R * C * (2 * res + 4) + 4 * C * vecs, "flops": R * C * 12}
    new, kv = _lengths(c)
    T, H, KH, D = sum(new), c["heads"], c["kv_heads"], c["hd"]
    if c["kind"] == "rope":
        return {"bytes": 2 * 2 * T * (H + 2 * KH) * D + 4 * c["rot"], "flops": 3 * T * (H + KH) * c["rot"]}
    pairs, keys = 0, 0
    for n, L in zip(new, kv):
        pairs += _pairs(n, L, c["causal"], c["window"])
        keys += min(L, n + c["window"] - 1) if c["window"] else L
    return {"bytes": 2 * 2 * T * H * D + 2 * 2 * keys * KH * D + (4 * T * H if c["lse"] else 0), "flops": 4 * pairs * H * D}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "rope": _exact_rope, "attn": _exact_attn}[case["kind"]](s)


def _exact_norm(s):
    c = s["case"]

    def norm(v, at):
        if c[at] == "none":
            return v
        d = v - v.sum(1, keepdim=True) / c["C"] if c[at] == "layer" else v
        out = d / (d.pow(2).sum(1, keepdim=True) / c["C"] + 1e-6).sqrt() * s[at + "_w"].double()
        return out + s[at + "_b"].double() if s[at + "_b"] is not None else out

    z = s["scale"] * norm(s["h"].double(), "post")
    if s["gate"] is not None:
        rows = s["gate"].double()
        z = z * (rows.repeat_interleave(s["per"], 0)[:c["R"]] if s["per"] else rows)
    r = s["x"].double() + z
    return {"r": r, "y": norm(r, "pre")}


def _exact_rope(s):
    c = s["case"]
    H, KH, D, rot = c["heads"], c["kv_heads"], c["hd"], c["rot"]
    f, amp = _freqs(c).cuda(), _rope_scale(c)
    k, v = s["k"].double(), s["v"].double()
    new, kv = _lengths(c)
    q, row = [], 0
    for b, (n, L) in enumerate(zip(new, kv)):
        x = s["qkv"][row:row + n].double().view(n, H + 2 * KH, D)
        row += n
        pos = torch.arange(L - n, L, device="cuda")
        turn = torch.polar(torch.full((n, rot // 2), amp, dtype=torch.float64, device="cuda"), pos.double()[:, None] * f)
        z = x[:, :H + KH, :rot]
        half = c["layout"] == "half"
        pair = torch.complex(z[..., :rot // 2], z[..., rot // 2:]) if half else torch.complex(z[..., 0::2], z[..., 1::2])
        pair = pair * turn[:, None]
        rotated = torch.cat([pair.real, pair.imag], -1) if half else torch.view_as_real(pair).flatten(-2)
        z = torch.cat([rotated, x[:, :H + KH, rot:]], -1)
        q.append(z[:, :H])
        for page in range((L - n) // PAGE, (L - 1) // PAGE + 1):
            a, e = max(L - n, page * PAGE), min(L, (page + 1) * PAGE)
            at, rows = int(s["table"][b, page]), slice(a - (L - n), e - (L - n))
            k[at, :, a - page * PAGE:e - page * PAGE] = z[rows, H:].transpose(0, 1)
            v[at, :, a - page * PAGE:e - page * PAGE] = x[rows, H + KH:].transpose(0, 1)
    return {"q": torch.cat(q), "k": k, "v": v}


def _exact_attn(s):
    c = s["case"]
    H, KH, D = c["heads"], c["kv_heads"], c["hd"]
    G = H // KH
    new, kv = _lengths(c)
    y = torch.zeros(sum(new), H, D, dtype=torch.float64, device="cuda")
    lse = torch.full((sum(new), H), float("-inf"), dtype=torch.float64, device="cuda")
    row = 0
    for b, (n, L) in enumerate(zip(new, kv)):
        rows = slice(row, row + n)
        row += n
        if L == 0:
            continue
        pages = s["table"][b, :(L + PAGE - 1) // PAGE].long()
        pos = torch.arange(L - n, L, device="cuda")[:, None]
        j = torch.arange(L, device="cuda")[None]
        off = torch.zeros(n, L, dtype=torch.bool, device="cuda")
        if c["causal"]:
            off |= j > pos
        if c["window"]:
            off |= j <= pos - c["window"]
        for h in range(KH):
            k = s["k"][pages, h].reshape(-1, D)[:L].double()
            v = s["v"][pages, h].reshape(-1, D)[:L].double()
            z = torch.einsum("ngd,ld->gnl", s["q"][rows, h * G:(h + 1) * G].double(), k) * s["scale"]
            z = z.masked_fill(off, float("-inf"))
            lse[rows, h * G:(h + 1) * G] = torch.logsumexp(z, -1).t()
            top = z.max(-1, keepdim=True).values.clamp_min(-1e300)
            w = (z - top).exp()
            w = w / w.sum(-1, keepdim=True).clamp_min(1e-300)
            y[rows, h * G:(h + 1) * G] = torch.einsum("gnl,ld->ngd", w, v)
    return {"y": y, "lse": lse} if c["lse"] else {"y": y}
