"""Timed cases: the operators of a decoder step that checks drafted tokens.

  w4      products of a few tokens' rows with weights of 4 bits and a scale per group
  ruled   attention over a paged cache with score rules: a tanh cap, a bias by distance, a prefix
          that all see, a tree of drafted tokens
  logits  penalties for repeated tokens, bias, temperature and grammar mask on logits, with the
          best token and the log of the sum of exponentials
  accept  the path through each tree that the model's own choices confirm, and its keys and values
          moved to the places that follow one another

``prepare`` draws a case's inputs on the GPU, ``run`` is one pass: the plain form in 32 bits, or
(``own``) the calls that a user makes.  ``exact`` is the definition in 64 bits.  Lengths of a ragged
batch follow from the case alone, so that ``work`` can count them.
"""
import math
import random

import torch

own = False
_ctx = None


def _w4(name, M, K, N, group, zeros, bias, act, res, out):
    return {"name": name, "kind": "w4", "M": M, "K": K, "N": N, "group": group, "zeros": zeros, "bias": bias, "act": act,
            "res": res, "out": out}


def _ruled(name, B, n, lo, hi, heads, kv_heads, hd, cap=0.0, slopes=False, prefix=0, tree=False, window=0, page=64, lse=False):
    return {"name": name, "kind": "ruled", "B": B, "n": n, "kv_min": lo, "kv_max": hi, "heads": heads, "kv_heads": kv_heads,
            "hd": hd, "cap": cap, "slopes": slopes, "prefix": prefix, "tree": tree, "window": window, "page": page, "lse": lse}


def _logits(name, R, V, dtype, seen, bias, masked, store):
    return {"name": name, "kind": "logits", "R": R, "V": V, "dtype": dtype, "seen": seen, "bias": bias, "masked": masked,
            "store": store}


def _accept(name, B, wide, deep, layers, kv_heads, hd, page):
    return {"name": name, "kind": "accept", "B": B, "wide": wide, "deep": deep, "layers": layers, "kv_heads": kv_heads, "hd": hd,
            "page": page}


def listed():
    return [
        # one token of one request through a small projection: latency
        _w4("w4_one", 1, 2048, 2048, 128, False, False, "none", False, "bf16"),
        # the up projection of an MLP for 16 requests, zero points, fine groups
        _w4("w4_b16", 16, 4096, 14336, 64, True, True, "relu", False, "bf16"),
        # drafted tokens of 4 requests, 15 or so each, through the down projection and onto the residual stream
        _w4("w4_drafts", 61, 14336, 4096, 128, True, False, "none", True, "bf16"),
        # a tree of 4 drafted tokens of one short request, few heads: latency
        _ruled("tree_short", 1, 4, 300, 300, 12, 12, 64, tree=True, page=16),
        # trees of 24 drafted tokens, 16 requests of very different lengths
        _ruled("tree_b16", 16, 24, 1000, 12000, 32, 8, 128, tree=True),
        # one token of each of 48 requests, scores capped
        _ruled("capped_b48", 48, 1, 400, 12000, 32, 8, 128, cap=50.0),
        # a prompt whose bias falls with the distance, no rotary positions
        _ruled("distance_prompt", 1, 4095, 4095, 4095, 32, 32, 64, slopes=True),
        # prompts that begin with a prefix seen by all (an image's tokens), capped, sliding window
        _ruled("prefix_chunks", 4, 1500, 1600, 4000, 16, 8, 128, cap=30.0, prefix=577, window=2048, page=32, lse=True),
        # the greedy tokens of 4 requests from 16-bit logits: nothing but the best token is asked for, latency
        _logits("best_b4", 4, 32000, "bf16", 100, "none", False, False),
        # 64 requests that sample, long answers, grammars, a bias for all, an odd vocabulary
        _logits("grammar_b64", 64, 128001, "f32", 3000, "shared", True, True),
        # the tree of one request's drafts checked, two layers' caches: latency
        _accept("accept_one", 1, 3, 2, 2, 12, 64, 16),
        # trees of 64 requests' drafts checked, four layers' caches
        _accept("accept_b64", 64, 6, 4, 4, 8, 128, 64),
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(round(v / step)) * step)


def _draw(rng):
    kind = rng.choice(["w4", "w4", "ruled", "ruled", "ruled", "logits", "logits", "accept"])
    if kind == "w4":
        group = rng.choice([32, 64, 128])
        return _w4("", _log(rng, 1, 64), _log(rng, 256, 16384, group), _log(rng, 64, 16384, 8), group, rng.random() < 0.5,
                   rng.random() < 0.3, rng.choice(["none", "none", "relu"]), rng.random() < 0.3, rng.choice(["bf16", "bf16", "f32"]))
    if kind == "logits":
        return _logits("", _log(rng, 1, 512), _log(rng, 1000, 260000), rng.choice(["f32", "f32", "bf16"]),
                       rng.choice([0, _log(rng, 1, 8000)]), rng.choice(["none", "shared", "rows"]), rng.random() < 0.5,
                       rng.random() < 0.7)
    if kind == "accept":
        deep = rng.randint(1, 6)
        wide = rng.randint(deep + 1, max(deep + 1, 63 // deep))
        return _accept("", _log(rng, 1, 64), min(wide, 63 // deep), deep, rng.randint(1, 4), rng.choice([1, 2, 4, 8]),
                       rng.choice([64, 128]), rng.choice([16, 32, 64, 128]))
    kv_heads, hd = rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 6, 8])
    form = rng.choice(["tree", "tree", "one", "chunk"])
    if form == "tree":
        B, n = _log(rng, 1, 32), rng.randint(2, 64)
        hi = n + _log(rng, 1, 12000)
    elif form == "one":
        B, n = _log(rng, 1, 64), 1
        hi = n + _log(rng, 1, 60000 if B <= 2 else 8000)
    else:
        n = _log(rng, 2, 3000)
        B = max(1, min(16, _log(rng, 1, max(1, 4000 // n))))
        hi = n + _log(rng, 1, 4000)
    lo = max(n, hi // rng.choice([1, 2, 10, 30]))
    rules = rng.choice([("cap",), ("slopes",), ("prefix",), ("cap", "slopes"), ("cap", "prefix")])
    if form == "tree":
        rules = rng.choice([(), (), ("cap",), ("slopes",)])
    return _ruled("", B, n, lo, hi, heads, kv_heads, hd, cap=rng.choice([20.0, 30.0, 50.0]) if "cap" in rules else 0.0,
                  slopes="slopes" in rules, prefix=_log(rng, 1, hi) if "prefix" in rules else 0, tree=form == "tree",
                  window=rng.choice([0, 0, 0, 100, 1000]), page=rng.choice([16, 32, 64, 128]), lse=rng.random() < 0.3)


def draw(rng):
    """One more case of the listed ranges, no more work than the largest of its kind."""
    while True:
        c = _draw(rng)
        del c["name"]
        most = [work(x) for x in listed() if x["kind"] == c["kind"]]
        w = work(c)
        if w["bytes"] > max(m["bytes"] for m in most) or w["flops"] > max(m["flops"] for m in most):
            continue
        # the plain form holds all scores of a padded batch
        if c["kind"] == "ruled" and c["B"] * c["heads"] * c["n"] * c["kv_max"] > 32 * 4096 * 4096:
            continue
        return c


# ---------------------------------------------------------------------------
# lengths
# ---------------------------------------------------------------------------
def _spread(b, lo, hi):
    """Lengths spread evenly over their logarithm."""
    return max(1, int(round(lo * (hi / lo) ** ((b * 0.6180339887498949) % 1.0))))


def _lengths(c):
    """New tokens and cached tokens (the new ones among them) of each sequence."""
    if c["kind"] == "accept":
        n = 1 + c["wide"] * c["deep"]
        return [n] * c["B"], [n + _spread(b, 40, 250) for b in range(c["B"])]
    new, kv = [], []
    for b in range(c["B"]):
        kv.append(_spread(b, c["kv_min"], c["kv_max"]) if c["B"] > 1 else c["kv_max"])
        m = c["n"] if b == 0 or c["n"] <= 2 else max(1, int(round(c["n"] * (0.5 + 0.5 * ((b * 0.7548776662466927) % 1.0)))))
        new.append(min(m, kv[-1]))
    return new, kv


def _seen_lengths(c):
    return [0 if not c["seen"] or r % 7 == 3 else _spread(r, max(1, c["seen"] // 10), c["seen"]) for r in range(c["R"])]


def _parents(c):
    """Each new token's parent in its sequence's tree: -1 for the first."""
    rng = random.Random(c["B"] * 1000 + c["n"])
    new, _ = _lengths(c)
    return [[-1] + [rng.randint(max(0, i // 3 - 2), i - 1) for i in range(1, n)] for n in new]


def _ancestors(parents):
    out = []
    for p in parents:
        bits = []
        for i, up in enumerate(p):
            bits.append((bits[up] if up >= 0 else 0) | 1 << i)
        out += bits
    return out


def _signed(v):
    return v - (1 << 64) if v >> 63 else v


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _table(c, g, new, kv):
    """A shuffled page table of the sequences, and the pages of the pool."""
    page = c["page"]
    need = [(L + page - 1) // page for L in kv]
    pages, width = sum(need) + 3, max(need)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((c["B"], width), -1, dtype=torch.int32, device="cuda")
    cols = torch.arange(width, device="cuda")
    needed = torch.tensor(need, device="cuda")
    live = cols[None] < needed[:, None]
    table[live] = order[((torch.cumsum(needed, 0) - needed)[:, None] + cols[None])[live]]
    return table, live, pages


def prepare(case, seed):
    global _ctx
    s = {"case": case}
    {"w4": _prepare_w4, "ruled": _prepare_ruled, "logits": _prepare_logits, "accept": _prepare_accept}[case["kind"]](s, case, _gen(seed))
    if own:
        from paper_2511_19457_gb300 import sparoa as sp
        if _ctx is None:
            _ctx = sp.Context(0)
        s["ctx"], s["sp"] = _ctx, sp
        _prepare_own(s, case)
    return s


def _prepare_w4(s, c, g):
    M, K, N, G = c["M"], c["K"], c["N"], c["group"]
    chan = torch.exp(0.3 * torch.randn(K, generator=g, device="cuda"))
    s["x"] = (torch.randn(M, K, generator=g, device="cuda") * chan).to(torch.bfloat16)
    # two codes a byte, the even column's in the low half
    s["codes"] = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s["scales"] = ((torch.rand(N, K // G, generator=g, device="cuda") + 0.5) * (0.25 / math.sqrt(K))).to(torch.bfloat16)
    s["zeros"] = torch.randint(5, 11, (N, K // G), generator=g, device="cuda", dtype=torch.uint8) if c["zeros"] else None
    s["bias"] = torch.randn(N, generator=g, device="cuda") * 0.1 if c["bias"] else None
    s["res"] = torch.randn(M, N, generator=g, device="cuda").to(torch.bfloat16) if c["res"] else None


def _prepare_ruled(s, c, g):
    H, KH, D, page = c["heads"], c["kv_heads"], c["hd"], c["page"]
    new, kv = _lengths(c)
    T = sum(new)
    table, live, pages = _table(c, g, new, kv)
    s["table"] = table
    s["q_start"] = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
    s["kv_len"], s["max_q"] = _ints(kv), max(new)
    s["q"] = (torch.randn(T, H, D, generator=g, device="cuda") * 1.5).to(torch.bfloat16)
    s["k"] = torch.randn(pages, KH, page, D, generator=g, device="cuda").to(torch.bfloat16)
    s["v"] = torch.randn(pages, KH, page, D, generator=g, device="cuda").to(torch.bfloat16)
    # what no token has been written to holds anything
    pos = torch.arange(table.shape[1], device="cuda")[:, None] * page + torch.arange(page, device="cuda")
    unused = torch.ones(pages, page, dtype=torch.bool, device="cuda")
    unused[table[live].long()] = ~((pos[None] < s["kv_len"][:, None, None]) & live[..., None])[live]
    s["k"].masked_fill_(unused[:, None, :, None], float("nan"))
    s["v"].masked_fill_(unused[:, None, :, None], float("nan"))
    s["scale"] = 1.0 / math.sqrt(D)
    h = torch.arange(1, H + 1, device="cuda", dtype=torch.float32)
    s["slopes"] = torch.exp2(-8.0 * h / H) if c["slopes"] else None
    s["prefix"] = _ints([min(L, max(1, c["prefix"] - 13 * b)) for b, L in enumerate(kv)]) if c["prefix"] else None
    s["tree"] = torch.tensor([_signed(v) for v in _ancestors(_parents(c))], device="cuda") if c["tree"] else None


def _prepare_logits(s, c, g):
    R, V = c["R"], c["V"]
    x = torch.randn(R, V, generator=g, device="cuda") * 2.5
    # a few tokens that stand out
    x += 12.0 * (torch.rand(R, V, generator=g, device="cuda") > 1.0 - 20.0 / V)
    s["logits"] = x if c["dtype"] == "f32" else x.to(torch.bfloat16)
    lens = _seen_lengths(c)
    s["seen_start"] = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
    total = sum(lens)
    # answers repeat themselves: squares lean to the low token numbers
    u = torch.rand(max(total, 1), generator=g, device="cuda", dtype=torch.float64)
    s["seen"] = (u * u * u * V).long().clamp_max(V - 1).to(torch.int32)[:total]
    par = torch.rand(R, 4, generator=g, device="cuda")
    s["penalties"] = torch.stack([1.0 + 0.3 * par[:, 0], par[:, 1] - 0.2, 0.5 * par[:, 2], 0.5 + par[:, 3]], 1)
    s["bias"] = None
    if c["bias"] != "none":
        b = torch.randn(R if c["bias"] == "rows" else 1, V, generator=g, device="cuda")
        s["bias"] = b * (torch.rand(b.shape, generator=g, device="cuda") < 0.1)
    s["allowed"] = None
    if c["masked"]:
        words = torch.randint(-2 ** 31, 2 ** 31, (R, (V + 31) // 32), generator=g, device="cuda", dtype=torch.int64)
        words &= torch.randint(-2 ** 31, 2 ** 31, words.shape, generator=g, device="cuda", dtype=torch.int64)
        s["allowed"] = words.to(torch.int32)


def _prepare_accept(s, c, g):
    KH, D, page, B = c["kv_heads"], c["hd"], c["page"], c["B"]
    wide, deep = c["wide"], c["deep"]
    new, kv = _lengths(c)
    n = new[0]
    s["table"], _, pages = _table(c, g, new, kv)
    s["q_start"] = torch.arange(B + 1, dtype=torch.int32, device="cuda") * n
    s["kv_len"], s["max_q"] = _ints(kv), n
    s["k"] = [torch.randn(pages, KH, page, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(c["layers"])]
    s["v"] = [torch.randn(pages, KH, page, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(c["layers"])]
    # `wide` chains of `deep` drafted tokens behind the first token, level by level.  The chain that the
    # model follows, and how far, is such that no token's new place is another kept token's old one.
    parents = [-1] + [0] * wide + list(range(1, 1 + wide * (deep - 1)))
    s["tree"] = torch.tensor([_signed(v) for v in _ancestors([parents])], device="cuda").repeat(B)
    order = torch.rand(B, 32000, generator=g, device="cuda").argsort(1)[:, :n]
    chain = torch.randint(0, wide - deep + 1, (B,), generator=g, device="cuda")
    chain = torch.where(chain > 0, chain + deep - 1, 0)
    follows = torch.randint(0, deep + 1, (B,), generator=g, device="cuda")
    best = torch.randint(32000, 33000, (B, n), generator=g, device="cuda")
    at = torch.zeros(B, dtype=torch.long, device="cuda")
    row = torch.arange(B, device="cuda")
    for d in range(deep):
        to = 1 + d * wide + chain
        best[row, at] = torch.where(follows > d, order[row, to], best[row, at])
        at = to
    s["tokens"], s["best"] = order.reshape(-1).to(torch.int32), best.reshape(-1).to(torch.int32)


def _prepare_own(s, c):
    sp, kind = s["sp"], c["kind"]

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if kind == "w4":
        s["w"] = sp.W4(s["ctx"], s["codes"], s["scales"], s["zeros"])
        s["y"] = empty(c["M"], c["N"], dtype=torch.float32 if c["out"] == "f32" else torch.bfloat16)
    elif kind == "logits":
        s["rules"] = sp.LogitRules(seen_start=s["seen_start"] if c["seen"] else None, seen=s["seen"] if c["seen"] else None,
                                   penalties=s["penalties"], bias=s["bias"], allowed=s["allowed"])
        s["y"] = empty(c["R"], c["V"]) if c["store"] else None
        s["out"] = (empty(c["R"], dtype=torch.int32), empty(c["R"]))
    else:
        s["batch"] = sp.PagedBatch(s["q_start"], s["kv_len"], s["table"], max_q=s["max_q"])
        if kind == "ruled":
            s["cache"] = sp.KVCache(s["k"], s["v"])
            s["rules"] = sp.ScoreRules(cap=c["cap"], slopes=s["slopes"], prefix=s["prefix"], tree=s["tree"])
            s["y"] = torch.empty_like(s["q"])
            s["lse"] = empty(s["q"].shape[0], c["heads"]) if c["lse"] else None
        else:
            s["caches"] = [sp.KVCache(k, v) for k, v in zip(s["k"], s["v"])]
            s["out"] = [torch.empty_like(s["tokens"])] + [empty(c["B"], dtype=torch.int32) for _ in range(3)]


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"w4": _own_w4, "ruled": _own_ruled, "logits": _own_logits, "accept": _own_accept}[kind](s)
    return {"w4": _plain_w4, "ruled": _plain_ruled, "logits": _plain_logits, "accept": _plain_accept}[kind](s)


def _own_w4(s):
    c, sp = s["case"], s["sp"]
    sp.sparoa_gemm_w4(s["ctx"], s["x"], s["w"], s["y"], bias=s["bias"], act=sp.ACT_RELU if c["act"] == "relu" else sp.ACT_NONE,
                      residual=s["res"])
    return {"y": s["y"]}


def _own_ruled(s):
    c = s["case"]
    s["sp"].sparoa_ruled_attention(s["ctx"], s["q"], s["y"], s["cache"], s["batch"], s["rules"], scale=s["scale"],
                                   window=c["window"], lse=s["lse"])
    return {"y": s["y"]} if s["lse"] is None else {"y": s["y"], "lse": s["lse"]}


def _own_logits(s):
    best, lse = s["out"]
    s["sp"].sparoa_shape_logits(s["ctx"], s["logits"], s["rules"], y=s["y"], best=best, lse=lse)
    return {"best": best, "lse": lse} if s["y"] is None else {"y": s["y"], "best": best, "lse": lse}


def _own_accept(s):
    path, count, following, length = s["out"]
    s["sp"].sparoa_tree_accept(s["ctx"], s["tokens"], s["best"], s["tree"], s["caches"], s["batch"], path, count, following, length)
    return {"path": path, "count": count, "following": following, "length": length, "k": s["k"], "v": s["v"]}


def _plain_w4(s):
    c = s["case"]
    N, K = c["N"], c["K"]
    codes = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).view(N, K).float()
    zeros = s["zeros"].float()[..., None] if c["zeros"] else 8.0
    w = ((codes.view(N, -1, c["group"]) - zeros) * s["scales"].float()[..., None]).view(N, K)
    y = torch.matmul(s["x"].float(), w.t())
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["res"] is not None:
        y = y + s["res"].float()
    if c["act"] == "relu":
        y = y.clamp_min(0.0)
    return {"y": y if c["out"] == "f32" else y.to(torch.bfloat16)}


def _plain_ruled(s):
    c = s["case"]
    H, KH, D, page = c["heads"], c["kv_heads"], c["hd"], c["page"]
    G, B, n = H // KH, c["B"], s["max_q"]
    start = s["q_start"].long()
    new, L = (start[1:] - start[:-1])[:, None], s["kv_len"].long()[:, None]
    i = torch.arange(n, device="cuda")[None]
    at = (start[:-1, None] + i).clamp_max(s["q"].shape[0] - 1)
    q = s["q"][at].float().view(B, n, KH, G, D).permute(0, 2, 3, 1, 4).reshape(B, KH, G * n, D)
    width = s["table"].shape[1]
    table = s["table"].long().clamp_min(0)
    j = torch.arange(width * page, device="cuda")[None]
    there = (j < L)[:, None, :, None]

    def keys(pool):
        rows = pool[table].permute(0, 2, 1, 3, 4).reshape(B, KH, width * page, D).float()
        return torch.where(there, rows, 0.0)

    pos = L - new + i
    if c["tree"]:
        # each token's ancestors, itself among them; its position is its depth
        node = torch.arange(64, device="cuda")
        bits = (s["tree"][at][..., None] >> node) & 1
        own_bit = node == i[..., None]
        bits = torch.where(own_bit, 1, torch.where(node < i[..., None], bits, 0))
        pos = L - new + bits.sum(-1) - 1
        index = j - (L - new)
        drafted = (index >= 0) & (index < 64)
        pick = index.clamp(0, 63)[:, None].expand(B, n, -1)
        ancestor = bits.gather(2, pick) == 1
        behind = bits.flip(-1).cumsum(-1).flip(-1).gather(2, pick) - 1  # ancestors after this one
        keep = torch.where(drafted[:, None], ancestor, (index < 0)[:, None])
        distance = torch.where(drafted[:, None], behind, pos[..., None] - j[:, None])
    else:
        keep = j[:, None] <= pos[..., None]
        if c["prefix"]:
            keep = keep | (j < s["prefix"].long()[:, None])[:, None]
        distance = pos[..., None] - j[:, None]
    keep = keep & (j < L)[:, None]
    if c["window"]:
        keep = keep & (distance < c["window"])
    x = torch.matmul(q, keys(s["k"]).transpose(-1, -2)).mul_(s["scale"]).view(B, KH, G, n, -1)
    if c["cap"]:
        x = x.div_(c["cap"]).tanh_().mul_(c["cap"])
    if c["slopes"]:
        x -= s["slopes"].view(1, KH, G, 1, 1) * distance.abs().float()[:, None, None]
    x.masked_fill_(~keep[:, None, None], float("-inf"))
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)
    p = x.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, KH, G * n, -1), keys(s["v"])).view(B, KH, G, n, D)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, n, H, D)
    valid = i < new
    y = o[valid].to(torch.bfloat16)
    if not c["lse"]:
        return {"y": y}
    lse = (m + total.log())[..., 0].permute(0, 3, 1, 2).reshape(B, n, H)
    return {"y": y, "lse": lse[valid]}


def _plain_logits(s):
    c = s["case"]
    R, V = c["R"], c["V"]
    y = s["logits"].float()
    rep, presence, frequency, temperature = (s["penalties"][:, i:i + 1] for i in range(4))
    if c["seen"]:
        start = s["seen_start"].long()
        row = torch.searchsorted(start[1:].contiguous(), torch.arange(s["seen"].numel(), device="cuda"), right=True)
        count = torch.zeros(R, V, device="cuda")
        count.index_put_((row, s["seen"].long()), torch.ones((), device="cuda"), accumulate=True)
        less = torch.where(y > 0, y / rep, y * rep) - presence - frequency * count
        y = torch.where(count > 0, less, y)
    if s["bias"] is not None:
        y = y + s["bias"]
    y = y * (1.0 / temperature)
    if c["masked"]:
        v = torch.arange(V, device="cuda")
        y = torch.where((s["allowed"][:, v // 32] >> (v % 32)) & 1 == 1, y, float("-inf"))
    m = y.amax(1, keepdim=True)
    first = torch.where(y == m, torch.arange(V, device="cuda"), V).amin(1)
    best = torch.where(m[:, 0] > float("-inf"), first, -1).to(torch.int32)
    shift = torch.where(m > float("-inf"), m, 0.0)
    lse = (shift + (y - shift).exp().sum(1, keepdim=True).log())[:, 0]
    return {"y": y, "best": best, "lse": lse} if c["store"] else {"best": best, "lse": lse}


def _plain_accept(s):
    c = s["case"]
    B, n, page = c["B"], s["max_q"], c["page"]
    node = torch.arange(n, device="cuda")
    tree = s["tree"].view(B, n)
    above = tree & ~(torch.ones_like(node) << node)  # ancestors without the token itself
    tokens, best = s["tokens"].view(B, n), s["best"].view(B, n)
    row = torch.arange(B, device="cuda")
    at = torch.zeros(B, dtype=torch.long, device="cuda")
    live = torch.ones(B, dtype=torch.bool, device="cuda")
    path = torch.full((B, n), -1, dtype=torch.long, device="cuda")
    following = torch.full((B,), -1, dtype=torch.long, device="cuda")
    for k in range(n):
        path[:, k] = torch.where(live, at, -1)
        following = torch.where(live, best[row, at].long(), following)
        child = (above == tree[row, at][:, None]) & (tokens == best[row, at][:, None])
        first = torch.where(child, node, n).amin(1)
        live = live & (first < n)
        at = torch.where(live, first, at)
    count = (path >= 0).sum(1)
    base = (s["kv_len"] - n).long()[:, None]
    b, k = torch.nonzero(path >= 0, as_tuple=True)
    src, dst = (base + path)[b, k], (base + node)[b, k]
    p0, p1 = s["table"].long()[b, src // page], s["table"].long()[b, dst // page]
    for pool in s["k"] + s["v"]:
        pool[p1, :, dst % page] = pool[p0, :, src % page]
    return {"path": path.view(-1).to(torch.int32), "count": count.to(torch.int32), "following": following.to(torch.int32),
            "length": (base[:, 0] + count).to(torch.int32), "k": s["k"], "v": s["v"]}


# ---------------------------------------------------------------------------
# the work of a pass
# ---------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "w4":
        M, K, N, groups = c["M"], c["K"], c["N"], c["K"] // c["group"]
        out = 4 if c["out"] == "f32" else 2
        return {"bytes": N * K // 2 + N * groups * (3 if c["zeros"] else 2) + 2 * M * K + M * N * (out + (2 if c["res"] else 0)) +
                (4 * N if c["bias"] else 0), "flops": 2 * M * K * N}
    if c["kind"] == "logits":
        R, V = c["R"], c["V"]
        vals = R * V * ((4 if c["dtype"] == "f32" else 2) + (4 if c["store"] else 0))
        bias = {"none": 0, "shared": 4 * V, "rows": 4 * R * V}[c["bias"]]
        return {"bytes": vals + bias + (4 * R * ((V + 31) // 32) if c["masked"] else 0) + 4 * sum(_seen_lengths(c)) + 24 * R,
                "flops": 6 * R * V}
    new, kv = _lengths(c)
    if c["kind"] == "accept":
        # half of the drafted tokens' depth is followed
        moved = c["B"] * c["deep"] / 2
        return {"bytes": int(moved * c["layers"] * 2 * 2 * 2 * c["kv_heads"] * c["hd"]) + 16 * sum(new) + 16 * c["B"], "flops": 32 * sum(new)}
    T, H, KH, D = sum(new), c["heads"], c["kv_heads"], c["hd"]
    parents = _parents(c) if c["tree"] else None
    pairs, keys = 0, 0
    for b, (n, L) in enumerate(zip(new, kv)):
        pre = min(L, max(1, c["prefix"] - 13 * b)) if c["prefix"] else 0
        depth = []
        for i in range(n):
            if parents:
                up = parents[b][i]
                depth.append(depth[up] + 1 if up >= 0 else 1)
                total = L - n + depth[-1]
                pairs += min(total, c["window"]) if c["window"] else total
            else:
                p = L - n + i
                pairs += max(0, max(p + 1, pre) - (max(0, p + 1 - c["window"]) if c["window"] else 0))
        keys += min(L, n + c["window"] - 1) if c["window"] else L
    return {"bytes": 2 * 2 * T * H * D + 2 * 2 * keys * KH * D + (4 * T * H if c["lse"] else 0) + (8 * T if c["tree"] else 0),
            "flops": 4 * pairs * H * D}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"w4": _exact_w4, "ruled": _exact_ruled, "logits": _exact_logits, "accept": _exact_accept}[case["kind"]](s)


def _exact_w4(s):
    c = s["case"]
    y = torch.zeros(c["M"], c["N"], dtype=torch.float64, device="cuda")
    x = s["x"].double()
    for g in range(c["K"] // c["group"]):
        k0, k1 = g * c["group"], (g + 1) * c["group"]
        b = s["codes"][:, k0 // 2:k1 // 2].long()
        z = s["zeros"][:, g:g + 1].long() if c["zeros"] else 8
        a = x[:, k0:k1]
        part = a[:, 0::2] @ (b % 16 - z).double().t() + a[:, 1::2] @ (b // 16 - z).double().t()
        y += part * s["scales"][:, g].double()
    y = y if s["bias"] is None else y + s["bias"].double()
    y = y if s["res"] is None else y + s["res"].double()
    return {"y": torch.relu(y) if c["act"] == "relu" else y}


def _exact_ruled(s):
    c = s["case"]
    H, KH, D, page = c["heads"], c["kv_heads"], c["hd"], c["page"]
    G = H // KH
    new, kv = _lengths(c)
    y = torch.zeros(sum(new), H, D, dtype=torch.float64, device="cuda")
    lse = torch.full((sum(new), H), float("-inf"), dtype=torch.float64, device="cuda")
    parents = _parents(c) if c["tree"] else None
    row = 0
    for b, (n, L) in enumerate(zip(new, kv)):
        rows = slice(row, row + n)
        row += n
        pages = s["table"][b, :(L + page - 1) // page].long()
        j = torch.arange(L, device="cuda")[None]
        far = torch.arange(L - n, L, device="cuda")[:, None] - j
        off = far < 0
        if parents:
            up, dist = parents[b], [[-1] * n for _ in range(n)]
            depth = [0] * n
            for i in range(n):
                a, d = i, 0
                while a >= 0:
                    dist[i][a] = d
                    a, d = up[a], d + 1
                depth[i] = d - 1
            near = torch.tensor(dist, device="cuda")
            far = torch.tensor(depth, device="cuda")[:, None] + L - n - j
            far[:, L - n:] = near
            off = torch.zeros_like(far, dtype=torch.bool)
            off[:, L - n:] = near < 0
        elif c["prefix"]:
            off &= j >= min(L, max(1, c["prefix"] - 13 * b))
        if c["window"]:
            off |= far >= c["window"]
        for h in range(KH):
            k = s["k"][pages, h].reshape(-1, D)[:L].double()
            v = s["v"][pages, h].reshape(-1, D)[:L].double()
            z = torch.einsum("ngd,ld->gnl", s["q"][rows, h * G:(h + 1) * G].double(), k) * s["scale"]
            if c["cap"]:
                z = c["cap"] * torch.tanh(z / c["cap"])
            if c["slopes"]:
                z -= s["slopes"][h * G:(h + 1) * G].double()[:, None, None] * far.abs()
            z = z.masked_fill(off, float("-inf"))
            lse[rows, h * G:(h + 1) * G] = torch.logsumexp(z, -1).t()
            w = (z - z.max(-1, keepdim=True).values.clamp_min(-1e300)).exp()
            w = w / w.sum(-1, keepdim=True).clamp_min(1e-300)
            y[rows, h * G:(h + 1) * G] = torch.einsum("gnl,ld->ngd", w, v)
    return {"y": y, "lse": lse} if c["lse"] else {"y": y}


def _exact_logits(s):
    c = s["case"]
    R, V = c["R"], c["V"]
    y = torch.empty(R, V, dtype=torch.float64, device="cuda")
    start = s["seen_start"].tolist()
    par = s["penalties"].double().tolist()
    for r in range(R):
        x = s["logits"][r].double()
        rep, presence, frequency, temperature = par[r]
        if start[r + 1] > start[r]:
            token, count = torch.unique(s["seen"][start[r]:start[r + 1]].long(), return_counts=True)
            z = x[token]
            x[token] = torch.where(z > 0, z / rep, z * rep) - presence - frequency * count.double()
        if s["bias"] is not None:
            x += s["bias"][r if c["bias"] == "rows" else 0].double()
        x /= temperature
        if c["masked"]:
            bit = torch.arange(32, device="cuda", dtype=torch.int32)
            on = ((s["allowed"][r][:, None] >> bit) & 1).flatten()[:V] == 1
            x = x.masked_fill(~on, float("-inf"))
        y[r] = x
    out = {"best": y.argmax(1).to(torch.int32), "lse": torch.logsumexp(y, 1)}
    return {"y": y, **out} if c["store"] else out


def _exact_accept(s):
    c = s["case"]
    page, n = c["page"], 1 + c["wide"] * c["deep"]
    _, kv = _lengths(c)
    k, v = [t.clone() for t in s["k"]], [t.clone() for t in s["v"]]
    tokens, best, table = s["tokens"].tolist(), s["best"].tolist(), s["table"].tolist()
    path, count, following, length = [], [], [], []
    for b, L in enumerate(kv):
        at, way = 0, [0]
        while True:
            level = [at + c["wide"]] if at else list(range(1, c["wide"] + 1))
            to = [t for t in level if t < n and tokens[b * n + t] == best[b * n + at]]
            if not to:
                break
            at = to[0]
            way.append(at)
        for to, of in enumerate(way):
            (sp_, so), (dp, do) = divmod(L - n + of, page), divmod(L - n + to, page)
            for pool, old in zip(k + v, s["k"] + s["v"]):
                pool[table[b][dp], :, do] = old[table[b][sp_], :, so]
        path += way + [-1] * (n - len(way))
        count.append(len(way))
        following.append(best[b * n + at])
        length.append(L - n + len(way))
    return {"path": _ints(path), "count": _ints(count), "following": _ints(following), "length": _ints(length), "k": k, "v": v}
