"""A decoder stack that answers from a paged key/value cache, on the library's operators.

Per layer, on the new tokens of all sequences at once ([T, C] rows, sequence after sequence):

    y   = N1(x)                                   sparoa_add_norm (of the layer before)
    qkv = y Wqkv                                  sparoa_gemm
    q, cache <- rotary positions of qkv           sparoa_rope_append
    a   = attention of q over the cache           sparoa_paged_attention
    r, y = x + g1 (a Wo), N2(r)                   sparoa_gemm, sparoa_add_norm
    h   = relu(y W1)                              sparoa_gemm, emits h's occupancy
    x, y = r + g2 (h W2), N1 of the next layer    sparoa_gemm by the threshold rule, sparoa_add_norm

The residual stream is fp32, everything between operators bf16.  ``Pages`` hands out the cache's
pages; a sequence holds its pages until it is freed.

With 4-bit weights (``group``) the products are sparoa_gemm_w4; with a cap of the scores or a bias by
distance (``cap``, ``slopes``), and over trees of drafted tokens, the attention is sparoa_ruled_attention.
Logits become tokens by sparoa_shape_logits.  ``check`` judges trees of drafted tokens in one step
(sparoa_tree_accept keeps the path that the model's own choices confirm); ``generate`` takes the drafts from a
function of the tokens so far.

    python -m paper_2511_19457_gb300.decoder      # a few prompts in chunks, then tokens one by one and by drafts
"""
from __future__ import annotations

import math

import torch

from . import sparoa as sp


class Pages:
    """Which pages of a cache a set of sequences holds."""

    def __init__(self, pages: int, page_size: int):
        self.page_size = page_size
        self.free = list(range(pages - 1, -1, -1))
        self.held: dict = {}     # sequence -> its pages, in order
        self.length: dict = {}   # sequence -> tokens in the cache

    def grow(self, seq, tokens: int):
        """Room for `tokens` more of a sequence (a new one, too); raises, and changes nothing, if the
        cache is full."""
        pages, length = self.held.get(seq, []), self.length.get(seq, 0) + tokens
        need = -(-length // self.page_size) - len(pages)
        if need > len(self.free):
            raise RuntimeError(f"cache full: {need} pages wanted, {len(self.free)} free")
        self.held[seq] = pages + [self.free.pop() for _ in range(need)]
        self.length[seq] = length

    def grow_all(self, seqs, new):
        """Room for new[i] more tokens of each of seqs; raises, and changes nothing, if the cache is full."""
        length: dict = {}
        for s, n in zip(seqs, new):
            length[s] = length.get(s, self.length.get(s, 0)) + n
        need = sum(-(-n // self.page_size) - len(self.held.get(s, [])) for s, n in length.items())
        if need > len(self.free):
            raise RuntimeError(f"cache full: {need} pages wanted, {len(self.free)} free")
        for s, n in zip(seqs, new):
            self.grow(s, n)

    def shrink_all(self, seqs, new):
        """Takes back the grow_all of the same tokens, if nothing came after it."""
        for s, n in zip(reversed(seqs), reversed(new)):
            length, pages = self.length[s] - n, self.held[s]
            keep = -(-length // self.page_size)
            self.free += reversed(pages[keep:])
            self.held[s], self.length[s] = pages[:keep], length
            if not length:
                self.release(s)

    def cut(self, seq, length: int):
        """Takes back what a sequence holds behind its first `length` tokens."""
        pages = self.held[seq]
        keep = -(-length // self.page_size)
        self.free += reversed(pages[keep:])
        self.held[seq], self.length[seq] = pages[:keep], length

    def release(self, seq):
        """Takes a sequence's pages back, if it has any."""
        self.free += reversed(self.held.pop(seq, []))
        self.length.pop(seq, None)

    def batch(self, seqs, new, device="cuda") -> sp.PagedBatch:
        """The new[i] last tokens of each of seqs, grown already."""
        table = [self.held[s] for s in seqs]
        width = max(len(t) for t in table)
        start = [0]
        for n in new:
            start.append(start[-1] + n)
        ints = [start, [self.length[s] for s in seqs], [t + [-1] * (width - len(t)) for t in table]]
        lists = [torch.tensor(v, dtype=torch.int32).to(device) for v in ints]
        return sp.PagedBatch(*lists, max_q=max(new))


def ancestors(parents):
    """Ancestor bits of a tree's tokens (its own among them) from each token's parent, -1 for none; parents
    come first."""
    if len(parents) > 64:
        raise ValueError("a tree of more than 64 tokens")
    bits: list = []
    for i, p in enumerate(parents):
        if not -1 <= p < i:
            raise ValueError(f"parent {p} of token {i}")
        bits.append((bits[p] if p >= 0 else 0) | 1 << i)
    return bits


class Decoder:
    """cap: attention scores s become cap tanh(s / cap); slopes (fp32 [heads]): a bias by distance instead of rotary
    positions; group: products with 4-bit weights, a scale for `group` columns."""

    def __init__(self, ctx: sp.Context, layers=2, dim=512, heads=8, kv_heads=2, head_dim=64, hidden=1024, vocab=1000,
                 pages=256, page_size=64, rope: sp.Rope | None = None, seed=0, device="cuda", cap=0.0, slopes=None,
                 group: int | None = None):
        g = torch.Generator().manual_seed(seed)

        def weight(n, k):
            w = (torch.randn(n, k, generator=g) / math.sqrt(k)).to(torch.bfloat16).to(device)
            return w if group is None else sp.W4.quantise(ctx, w, group)

        def gamma(shift):
            return (shift + 0.1 * torch.randn(dim, generator=g)).to(device)

        self.ctx, self.dim, self.heads, self.kv_heads, self.head_dim = ctx, dim, heads, kv_heads, head_dim
        self.embed = torch.randn(vocab, dim, generator=g).to(torch.bfloat16).to(device)
        width = (heads + 2 * kv_heads) * head_dim
        self.layers = [{"qkv": weight(width, dim), "o": weight(dim, heads * head_dim), "w1": weight(hidden, dim),
                        "w2": weight(dim, hidden), "n1": sp.norm("rms", gamma(1.0)), "n2": sp.norm("rms", gamma(1.0)),
                        "g1": gamma(0.5), "g2": gamma(0.5),
                        "cache": sp.KVCache.empty(pages, kv_heads, page_size, head_dim, device)} for _ in range(layers)]
        self.last = sp.norm("rms", gamma(1.0))
        self.rope = rope or sp.Rope(0 if slopes is not None else head_dim, device=device)
        self.cap, self.slopes = cap, None if slopes is None else slopes.to(device)
        self.pages = Pages(pages, page_size)
        self.hidden = hidden

    def forward(self, tokens: torch.Tensor, seqs, new) -> torch.Tensor:
        """tokens int64 [T], below the vocabulary's size (check and generate look, this does not), new[i] of
        each of seqs one after the other, appended to their cached ones; returns the logits [T, vocab]
        (fp32).  A step that raises changes no sequence's length."""
        self.pages.grow_all(seqs, new)
        try:
            return self._forward(tokens, seqs, new)
        except BaseException:
            self.pages.shrink_all(seqs, new)  # (what was appended of this step is written over by the next)
            raise

    def check(self, drafts, seqs):
        """Judge drafted tokens.  drafts[i] = (tokens, parents) of seqs[i], the first token the last one that is
        settled (and not in the cache yet), the others drafted behind their parents (parents[0] = -1).
        Returns for each sequence its next tokens: the drafted ones that the model would have chosen itself
        (greedily), and the one that it chooses after them.  The cache keeps what is settled.  Where the model
        chooses nothing (no logit is a number above -infinity), that is an error, and the cache as it was."""
        if len(drafts) != len(seqs) or len(set(seqs)) != len(seqs):
            raise ValueError("check: a tree for each sequence, and no sequence twice")
        if not drafts:
            return []
        new = [len(t) for t, _ in drafts]
        bits = [b for _, parents in drafts for b in ancestors(parents)]
        if any(len(t) != len(p) or not t or p[0] != -1 for t, p in drafts):
            raise ValueError("check: a tree begins with the last settled token and has a parent for each token")
        self._known(t for tokens, _ in drafts for t in tokens)
        dev = self.embed.device
        flat = torch.tensor([t for tokens, _ in drafts for t in tokens], dtype=torch.int32).to(dev)
        tree = torch.tensor([b - (1 << 64) if b >> 63 else b for b in bits], dtype=torch.int64).to(dev)
        depth = [bin(b).count("1") - 1 for b in bits]
        before = [self.pages.length.get(s, 0) for s in seqs]
        self.pages.grow_all(seqs, new)
        try:
            at, positions = 0, []
            for start, n in zip(before, new):
                positions += [start + d for d in depth[at:at + n]]
                at += n
            batch = self.pages.batch(seqs, new, dev)
            logits = self._layers(flat.long(), batch, tree, torch.tensor(positions, dtype=torch.int32).to(dev))
            best, path = torch.empty_like(flat), torch.empty_like(flat)
            sp.sparoa_shape_logits(self.ctx, logits, best=best)
            count, following, length = (torch.empty(len(seqs), dtype=torch.int32, device=dev) for _ in range(3))
            sp.sparoa_tree_accept(self.ctx, flat, best, tree, [w["cache"] for w in self.layers], batch, path, count, following, length)
            self.ctx.sync()  # (reports device-side failures)
            ways, counts, after, lengths = path.tolist(), count.tolist(), following.tolist(), length.tolist()
            if min(after, default=0) < 0:
                raise ValueError("check: a sequence that no token may follow")
        except BaseException:
            self.pages.shrink_all(seqs, new)
            raise
        out, at = [], 0
        for (tokens, _), s, n, c, f, L in zip(drafts, seqs, new, counts, after, lengths):
            out.append([tokens[i] for i in ways[at + 1:at + c]] + [f])
            self.pages.cut(s, L)
            at += n
        return out

    def _known(self, tokens):
        """Raises for a token that has no embedding (its row would be looked up on the GPU all the same)."""
        for t in tokens:
            if not 0 <= t < self.embed.shape[0]:
                raise ValueError(f"token {t} of {self.embed.shape[0]}")

    def _forward(self, tokens, seqs, new):
        return self._layers(tokens, self.pages.batch(seqs, new, tokens.device))

    def _layers(self, tokens, batch, tree=None, positions=None):
        ctx, T, dev = self.ctx, tokens.numel(), tokens.device

        def rows(width, dtype=torch.bfloat16):
            return torch.empty(T, width, dtype=dtype, device=dev)

        x, y = self.embed[tokens].float(), rows(self.dim)
        r, o, h = rows(self.dim, torch.float32), rows(self.dim), rows(self.hidden)
        qkv, q = rows((self.heads + 2 * self.kv_heads) * self.head_dim), rows(self.heads * self.head_dim)
        a = torch.empty_like(q)
        occ = sp.OccupancyBuffer(T, self.hidden, dev)
        dense = sp.thresholds(force_path=1)  # (norm and attention outputs have no zeros to skip)
        rules = None
        if tree is not None or self.cap or self.slopes is not None:
            rules = sp.ScoreRules(cap=self.cap, slopes=self.slopes, tree=tree)

        def product(x, w, y, **kw):
            if isinstance(w, sp.W4):
                sp.sparoa_gemm_w4(ctx, x, w, y, **kw)
            else:
                sp.sparoa_gemm(ctx, x, w, y, thr=dense, **kw)

        sp.sparoa_add_norm(ctx, x, None, None, y, pre=self.layers[0]["n1"])
        for i, w in enumerate(self.layers):
            after = self.layers[i + 1]["n1"] if i + 1 < len(self.layers) else self.last
            product(y, w["qkv"], qkv)
            sp.sparoa_rope_append(ctx, qkv, q, w["cache"], batch, self.rope, positions)
            if rules is None:
                sp.sparoa_paged_attention(ctx, q, a, w["cache"], batch)
            else:
                sp.sparoa_ruled_attention(ctx, q, a, w["cache"], batch, rules)
            product(a, w["o"], o)
            sp.sparoa_add_norm(ctx, x, o, r, y, gate=w["g1"], pre=w["n2"])
            if isinstance(w["w2"], sp.W4):
                product(y, w["w1"], h, act=sp.ACT_RELU)
                product(h, w["w2"], o)
            else:
                product(y, w["w1"], h, act=sp.ACT_RELU, y_occ=occ)
                sp.sparoa_gemm(ctx, h, w["w2"], o, x_occ=occ)
            sp.sparoa_add_norm(ctx, r, o, x, y, gate=w["g2"], pre=after)
        logits = rows(self.embed.shape[0], torch.float32)
        sp.sparoa_gemm(ctx, y, self.embed, logits, thr=dense)
        return logits

    def generate(self, prompts, steps: int, chunk: int = 256, draft=None, penalties=None, bias=None, allowed=None):
        """Greedy tokens after each prompt (lists of token numbers): prompts in chunks of at most
        `chunk` tokens each, all sequences together, then one token of each at a time.  No prompts:
        no tokens; an empty prompt, which nothing can be said after, is refused.
          draft      a function of a sequence's tokens so far: (tokens, parents) that may come next, parents by
                     their number among them, -1 behind the last token; they are judged together (check), and
                     hold pages of the cache until they are
          penalties  (repetition, presence, frequency, temperature) of every sequence
          bias       fp32 [vocab] on the logits
          allowed    a function of a sequence's tokens so far: int32 [words], bit v % 32 of word v / 32 for
                     every token that may come next
        Drafts go with none of the three others."""
        if not all(prompts):
            raise ValueError("generate: a prompt without tokens")
        self._known(t for p in prompts for t in p)
        if draft is not None and not (penalties is None and bias is None and allowed is None):
            raise ValueError("generate: drafts are judged by the logits as they are")
        if not prompts:
            return []
        seqs = [object() for _ in prompts]
        try:
            return self._generate(seqs, prompts, steps, chunk, draft, penalties, bias, allowed)
        finally:
            for s in seqs:
                self.pages.release(s)

    def _choose(self, logits, texts, penalties, bias, allowed):
        """The best token of each row of logits behind its text."""
        dev = logits.device
        best = torch.empty(len(texts), dtype=torch.int32, device=dev)
        rules = None
        if not (penalties is None and bias is None and allowed is None):
            lists, words, each = {}, None, None
            if penalties is not None:
                start = [0]
                for t in texts:
                    start.append(start[-1] + len(t))
                lists = {"seen_start": torch.tensor(start, dtype=torch.int32).to(dev),
                         "seen": torch.tensor([v for t in texts for v in t], dtype=torch.int32).to(dev)}
                each = torch.tensor([penalties] * len(texts), dtype=torch.float32).to(dev)
            if allowed is not None:
                words = torch.stack([allowed(t) for t in texts]).to(dev)
            rules = sp.LogitRules(penalties=each, bias=bias, allowed=words, **lists)
        sp.sparoa_shape_logits(self.ctx, logits, rules, best=best)
        out = best.tolist()
        if min(out) < 0:
            raise ValueError("generate: a sequence that no token may follow")
        return out

    def _generate(self, seqs, prompts, steps, chunk, draft, penalties, bias, allowed):
        dev = self.embed.device
        at = [0] * len(prompts)
        out: list = [[] for _ in prompts]
        while any(a < len(p) for a, p in zip(at, prompts)) or min(len(t) for t in out) < steps:
            todo = [(i, p[a:a + chunk]) for i, (a, p) in enumerate(zip(at, prompts)) if a < len(p)]
            if not todo:  # all prompts are in the cache
                if draft is not None:
                    self._check_drafts(seqs, prompts, out, steps, draft)
                    continue
                todo = [(i, [t[-1]]) for i, t in enumerate(out)]
            tokens = torch.tensor([t for _, part in todo for t in part]).to(dev)
            new = [len(part) for _, part in todo]
            logits = self.forward(tokens, [seqs[i] for i, _ in todo], new)
            ends = [(row, i) for row, (i, part) in zip(torch.tensor(new).cumsum(0).sub(1).tolist(), todo)
                    if at[i] + len(part) >= len(prompts[i])]
            for i, part in todo:
                at[i] += len(part)
            if ends:
                rows = logits if len(ends) == logits.shape[0] else logits[torch.tensor([r for r, _ in ends]).to(dev)]
                texts = [prompts[i] + out[i] for _, i in ends]
                for (_, i), token in zip(ends, self._choose(rows, texts, penalties, bias, allowed)):
                    out[i].append(token)
        self.ctx.sync()  # (reports device-side failures)
        return [t[:steps] for t in out]

    def _check_drafts(self, seqs, prompts, out, steps, draft):
        todo = [i for i, t in enumerate(out) if len(t) < steps]
        drafts = []
        for i in todo:
            tokens, parents = draft(prompts[i] + out[i])
            drafts.append(([out[i][-1]] + list(tokens), [-1] + [p + 1 for p in parents]))
        for i, more in zip(todo, self.check(drafts, [seqs[i] for i in todo])):
            out[i] += more


def repeats(text, tokens=4, ways=2):
    """Drafts from the text itself: what followed its last token the latest `ways` times, `tokens` each."""
    out, parents = [], []
    places = [i for i in range(len(text) - 2, -1, -1) if text[i] == text[-1]][:ways]
    for i in places:
        for k, t in enumerate(text[i + 1:i + 1 + tokens]):
            parents.append(-1 if k == 0 else len(out) - 1)
            out.append(t)
    return out, parents


def main():
    ctx = sp.Context(0)
    model = Decoder(ctx)
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, 1000, (n,), generator=g).tolist() for n in (700, 1, 300, 64)]
    for p, t in zip(prompts, model.generate(prompts, 16)):
        print(f"{len(p)} tokens -> {t}")
    for p, t in zip(prompts, model.generate(prompts, 16, draft=repeats)):
        print(f"{len(p)} tokens, drafts -> {t}")
    for p, t in zip(prompts, model.generate(prompts, 16, penalties=(1.0, 1e4, 0.0, 1.0))):
        print(f"{len(p)} tokens, none twice -> {t}")
    ctx.close()


if __name__ == "__main__":
    main()
