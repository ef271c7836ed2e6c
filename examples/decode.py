"""Scores prompts and decodes from a one-layer attention model whose five
projections are ternary factors (random weights; ``python examples/decode.py``).

A step, for the new tokens of all users side by side:

    apply (q, k, v) -> rotary -> kv4_append -> kv4_attention -> apply (o) -> apply (head) -> token_logprobs

The cache holds K and V in 4 bits, in pages that users take as they grow.
"""
from __future__ import annotations

import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2607_13511_amd import binding


class Factors:
    def __init__(self, A, mu):
        self.m, self.n = A.shape
        self.f = binding.factorize(A, mu=mu, tau=1.0, block=64, iters=4)

    def __call__(self, X):
        """X (rows x n) times the factors' transpose; apply takes eight rows a call."""
        parts = [binding.apply(self.f.B_packed, self.f.C_packed, self.f.D, self.m, self.n, x.contiguous())
                 for x in X.split(binding.APPLY_MAX_BATCH)]
        return torch.cat(parts)


class Model:
    def __init__(self, width=256, heads=8, heads_kv=2, dim=64, vocab=1000, mu=1.5, seed=0):
        gen = torch.Generator().manual_seed(seed)

        def factors(m, n):
            return Factors((torch.randn((m, n), generator=gen) / math.sqrt(n)).cuda(), mu)

        self.heads, self.heads_kv, self.dim, self.vocab = heads, heads_kv, dim, vocab
        self.embedding = torch.randn((vocab, width), generator=gen).cuda()
        self.q, self.k, self.v = factors(heads * dim, width), factors(heads_kv * dim, width), factors(heads_kv * dim, width)
        self.o, self.head = factors(width, heads * dim), factors(vocab, width)
        freqs, self.amplitude = binding.rotary_frequencies(dim, 10000.0, "parts", 4.0, 2048)
        self.freqs = torch.from_numpy(freqs).cuda()


class Session:
    """Users' sequences in one cache of `pages` pages."""

    def __init__(self, model, users, pages=64, page_tokens=16, most_pages=16):
        self.model, self.page_tokens, self.most_pages = model, page_tokens, most_pages
        self.cache = binding.kv4_cache(pages, model.heads_kv, model.dim, page_tokens)
        self.free = list(range(pages))
        self.lens = [0] * users
        self.table = torch.full((users, most_pages), -1, dtype=torch.int32)

    def _grow(self, news):
        pages = [(-(-have // self.page_tokens), -(-(have + n) // self.page_tokens)) for have, n in zip(self.lens, news)]
        wanted = 0
        for u, (have, need) in enumerate(pages):      # nothing is taken unless all users have room
            wanted += need - have
            if need > self.most_pages or wanted > len(self.free):
                raise RuntimeError(f"user {u}: no page left for {self.lens[u] + news[u]} tokens")
        for u, (have, need) in enumerate(pages):
            self.lens[u] += news[u]
            for i in range(have, need):
                self.table[u, i] = self.free.pop()

    def step(self, tokens, targets=None, top=5):
        """New tokens of each user (a list of lists); returns the last stage's
        ``TokenLogprobs`` for every one of them and what led to it."""
        m, news = self.model, [len(t) for t in tokens]
        self._grow(news)
        starts = [sum(news[:u]) for u in range(len(news) + 1)]
        positions = [self.lens[u] - news[u] + i for u in range(len(news)) for i in range(news[u])]
        table, T = self.table.cuda(), starts[-1]
        lens = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        st = torch.tensor(starts, dtype=torch.int32, device="cuda")
        pos = torch.tensor(positions, dtype=torch.int64, device="cuda")
        x = m.embedding[torch.tensor([t for ts in tokens for t in ts], device="cuda")]
        q0, k0 = m.q(x).view(T, m.heads, m.dim), m.k(x).view(T, m.heads_kv, m.dim)
        v = m.v(x).view(T, m.heads_kv, m.dim)
        q, k = binding.rotary(q0, k0, pos, m.freqs, amplitude=m.amplitude)
        binding.kv4_append(self.cache, k, v, table, lens, starts=st)
        att, lse = binding.kv4_attention(self.cache, q, table, lens, starts=st, max_new=max(news), max_len=max(self.lens))
        o = m.o(att.view(T, m.heads * m.dim))
        y = x + o
        logits = m.head(y)
        if targets is not None:
            targets = torch.tensor([t for ts in targets for t in ts], device="cuda")
        out = binding.token_logprobs(logits, targets, top=top)
        return out, dict(x=x, q0=q0, k0=k0, q=q, k=k, v=v, att=att, lse=lse, o=o, y=y, logits=logits,
                         positions=positions, starts=starts, table=table, lens=lens)


def main():
    model, gen = Model(), torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, model.vocab, (n,), generator=gen).tolist() for n in (70, 23, 1)]
    session = Session(model, len(prompts))
    out, _ = session.step(prompts, [p[1:] + [-1] for p in prompts])      # the last token's next one is not known
    scored = sum(len(p) - 1 for p in prompts)
    print(f"{scored} tokens scored, perplexity {math.exp(-float(out.logprob.sum()) / scored):.1f}")
    ends = [sum(len(p) for p in prompts[:u + 1]) - 1 for u in range(len(prompts))]
    last = out.top_ids[ends, 0].tolist()
    texts = [[t] for t in last]
    for _ in range(8):
        out, _ = session.step([[t] for t in last])
        last = out.top_ids[:, 0].tolist()
        for text, t in zip(texts, last):
            text.append(t)
    for u, text in enumerate(texts):
        print(f"user {u}: {session.lens[u]} tokens in the cache, decoded {text}")


if __name__ == "__main__":
    main()
