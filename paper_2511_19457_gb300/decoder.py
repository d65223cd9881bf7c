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

    python -m paper_2511_19457_gb300.decoder      # a few prompts in chunks, then tokens one by one
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


class Decoder:
    def __init__(self, ctx: sp.Context, layers=2, dim=512, heads=8, kv_heads=2, head_dim=64, hidden=1024, vocab=1000,
                 pages=256, page_size=64, rope: sp.Rope | None = None, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)

        def weight(n, k):
            return (torch.randn(n, k, generator=g) / math.sqrt(k)).to(torch.bfloat16).to(device)

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
        self.rope = rope or sp.Rope(head_dim, device=device)
        self.pages = Pages(pages, page_size)
        self.hidden = hidden

    def forward(self, tokens: torch.Tensor, seqs, new) -> torch.Tensor:
        """tokens int64 [T], new[i] of each of seqs one after the other, appended to their cached ones;
        returns the logits [T, vocab] (fp32).  A step that raises changes no sequence's length."""
        self.pages.grow_all(seqs, new)
        try:
            return self._forward(tokens, seqs, new)
        except BaseException:
            self.pages.shrink_all(seqs, new)  # (what was appended of this step is written over by the next)
            raise

    def _forward(self, tokens, seqs, new):
        ctx, T, dev = self.ctx, tokens.numel(), tokens.device
        batch = self.pages.batch(seqs, new, dev)

        def rows(width, dtype=torch.bfloat16):
            return torch.empty(T, width, dtype=dtype, device=dev)

        x, y = self.embed[tokens].float(), rows(self.dim)
        r, o, h = rows(self.dim, torch.float32), rows(self.dim), rows(self.hidden)
        qkv, q = rows((self.heads + 2 * self.kv_heads) * self.head_dim), rows(self.heads * self.head_dim)
        a = torch.empty_like(q)
        occ = sp.OccupancyBuffer(T, self.hidden, dev)
        dense = sp.thresholds(force_path=1)  # (norm and attention outputs have no zeros to skip)
        sp.sparoa_add_norm(ctx, x, None, None, y, pre=self.layers[0]["n1"])
        for i, w in enumerate(self.layers):
            after = self.layers[i + 1]["n1"] if i + 1 < len(self.layers) else self.last
            sp.sparoa_gemm(ctx, y, w["qkv"], qkv, thr=dense)
            sp.sparoa_rope_append(ctx, qkv, q, w["cache"], batch, self.rope)
            sp.sparoa_paged_attention(ctx, q, a, w["cache"], batch)
            sp.sparoa_gemm(ctx, a, w["o"], o, thr=dense)
            sp.sparoa_add_norm(ctx, x, o, r, y, gate=w["g1"], pre=w["n2"])
            sp.sparoa_gemm(ctx, y, w["w1"], h, act=sp.ACT_RELU, thr=dense, y_occ=occ)
            sp.sparoa_gemm(ctx, h, w["w2"], o, x_occ=occ)
            sp.sparoa_add_norm(ctx, r, o, x, y, gate=w["g2"], pre=after)
        logits = rows(self.embed.shape[0], torch.float32)
        sp.sparoa_gemm(ctx, y, self.embed, logits, thr=dense)
        return logits

    def generate(self, prompts, steps: int, chunk: int = 256):
        """Greedy tokens after each prompt (lists of token numbers): prompts in chunks of at most
        `chunk` tokens each, all sequences together, then one token of each at a time.  No prompts:
        no tokens; an empty prompt, which nothing can be said after, is refused."""
        if not all(prompts):
            raise ValueError("generate: a prompt without tokens")
        if not prompts:
            return []
        seqs = [object() for _ in prompts]
        try:
            return self._generate(seqs, prompts, steps, chunk)
        finally:
            for s in seqs:
                self.pages.release(s)

    def _generate(self, seqs, prompts, steps, chunk):
        dev = self.embed.device
        at = [0] * len(prompts)
        out: list = [[] for _ in prompts]
        while any(a < len(p) for a, p in zip(at, prompts)) or len(out[0]) < steps:
            todo = [(i, p[a:a + chunk]) for i, (a, p) in enumerate(zip(at, prompts)) if a < len(p)]
            if not todo:  # all prompts are in the cache
                todo = [(i, [t[-1]]) for i, t in enumerate(out)]
            tokens = torch.tensor([t for _, part in todo for t in part]).to(dev)
            new = [len(part) for _, part in todo]
            logits = self.forward(tokens, [seqs[i] for i, _ in todo], new)
            best = logits[torch.tensor(new).cumsum(0).to(dev) - 1].argmax(-1).tolist()
            for (i, part), token in zip(todo, best):
                at[i] += len(part)
                if at[i] >= len(prompts[i]):
                    out[i].append(token)
        self.ctx.sync()  # (reports device-side failures)
        return [t[:steps] for t in out]


def main():
    ctx = sp.Context(0)
    model = Decoder(ctx)
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, 1000, (n,), generator=g).tolist() for n in (700, 1, 300, 64)]
    for p, t in zip(prompts, model.generate(prompts, 16)):
        print(f"{len(p)} tokens -> {t}")
    ctx.close()


if __name__ == "__main__":
    main()
