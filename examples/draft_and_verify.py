#!/usr/bin/env python3
"""A small language model with attention out of this library's operators, decoding a batch of texts with drafted tokens over a paged cache.

A block is: queries, keys and values by one matrix in 4 bits (hbp_q4_mv), keys and values appended to the cache with their positions' rotation (hbp_paged_append),
attention of the new tokens over it (hbp_paged_attention), an output matrix, the norms around the residual sum (hbp_residual_norms), and the same for two matrices with an
activation.  The first block alone, with the output matrix behind it, drafts some tokens; then the whole model takes all of them at once, and hbp_verify_drafts says from
its logits which stand and what comes behind them.  What was cached of the others is written over by the next tokens.

    python examples/draft_and_verify.py [--width 256] [--blocks 3] [--vocabulary 2000] [--texts 4] [--tokens 40] [--drafts 4] [--temperature 0.8]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2504_08860_amd as H  # noqa: E402


class Q4:
    """A dense matrix rounded to 4 bits with group scales."""

    def __init__(self, w, group=32):
        codes, scales = H.hbp_q4_shapes(*w.shape, group)
        self.shape, self.group = tuple(w.shape), group
        self.codes = torch.empty(codes, dtype=torch.uint8, device="cuda")
        self.scales = torch.empty(scales, dtype=torch.float16, device="cuda")
        H.hbp_q4_pack(w, self.codes, self.scales, group=group)

    def __call__(self, x):
        y = x.new_empty(x.shape[0], self.shape[0])
        H.hbp_q4_mv(self.codes, self.scales, x.contiguous(), y, group=self.group)
        return y

    def values(self):
        return H.hbp_q4_unpack(self.codes, self.scales, self.shape[1], group=self.group)


class Model:
    def __init__(self, width=256, blocks=3, vocabulary=2000, heads=8, kv_heads=2, dtype=torch.float32, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
        self.width, self.vocabulary, self.heads, self.kv_heads, self.dtype, self.eps = width, vocabulary, heads, kv_heads, dtype, 1e-6
        self.head_dim = width // heads
        self.embedding = r(vocabulary, width).to(dtype)
        self.frequencies = (1000.0 ** (-torch.arange(self.head_dim // 2, device="cuda") / (self.head_dim // 2))).float()
        inner, size = 2 * width, width ** -0.5
        both = (heads + 2 * kv_heads) * self.head_dim
        self.qkv = [Q4(r(both, width) * size * 1.5) for _ in range(blocks)]
        self.out = [Q4(r(width, width) * size) for _ in range(blocks)]
        self.up, self.down = [Q4(r(inner, width) * size) for _ in range(blocks)], [Q4(r(width, inner) * inner ** -0.5) for _ in range(blocks)]
        self.norms = [[(1 + 0.1 * r(width)).to(dtype) for _ in range(4)] for _ in range(blocks)]
        self.w_in = (1 + 0.1 * r(width)).to(dtype)
        # (blocks behind the first one change little, so that its drafts are often right)
        self.scales = [0.7] + [0.25] * (blocks - 1)
        self.head = Q4(r(vocabulary, width) * size * 2.5)

    def cache(self, texts, most, page=16, seed=1):
        """Keys and values of each block for `texts` texts of up to `most` tokens, and the table of their pages, which were handed out in no order."""
        wide = -(-most // page)
        order = torch.randperm(texts * wide, generator=torch.Generator().manual_seed(seed)).int()
        shape = (texts * wide, self.kv_heads, page, self.head_dim)
        pages = [[torch.full(shape, float("nan"), dtype=self.dtype, device="cuda") for _ in range(2)] for _ in self.qkv]   # (nothing is in them yet)
        return pages, order.view(texts, wide).cuda()

    def __call__(self, tokens, starts, lengths, cache, blocks=None, most_new=None):
        """Logits [tokens, vocabulary] of new tokens (packed text by text at `starts`), which are appended to the cache: `lengths` tokens of each text with them."""
        pages, table = cache
        h = self.embedding[tokens]
        x = torch.empty_like(h)
        H.hbp_residual_norms(h, torch.zeros_like(h), h, x, w_pre=self.w_in, eps=self.eps)   # (no block yet: the norm alone)
        n, dim, q_wide, kv_wide = len(tokens), self.head_dim, self.heads * self.head_dim, self.kv_heads * self.head_dim
        for k in range(len(self.qkv) if blocks is None else blocks):
            q, key, value = (part.view(n, -1, dim) for part in self.qkv[k](x).split([q_wide, kv_wide, kv_wide], dim=1))
            keys, values = pages[k]
            H.hbp_paged_append(key, value, keys, values, table, starts, lengths, q=q, q_out=q, frequencies=self.frequencies)
            y = h.new_empty(n, self.heads, dim)
            H.hbp_paged_attention(q, keys, values, table, starts, lengths, y, softcap=30.0, most_new=most_new)
            between = dict(scale=self.scales[k], eps=self.eps)
            H.hbp_residual_norms(h, self.out[k](y.view(n, self.width)), h, x, w_post=self.norms[k][0], w_pre=self.norms[k][1], **between)
            H.hbp_residual_norms(h, self.down[k](torch.nn.functional.silu(self.up[k](x))), h, x, w_post=self.norms[k][2], w_pre=self.norms[k][3], **between)
        return self.head(x)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def decode(model, prompts, steps, drafts=4, temperature=0.0, seed=0):
    """`steps` new tokens (at least) behind each of `prompts` (lists of tokens): (the texts with them, drafts that stood, drafts that were made)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    texts, count = [list(p) for p in prompts], len(prompts)
    # (while the slowest text gets one token a round, another one may get all its drafts and one more, and a last round's lie behind that)
    most = max(len(p) for p in prompts) + (max(steps, 0) + 1) * (drafts + 1)
    cache = model.cache(count, most)
    heat = torch.full((count,), temperature, device="cuda")

    # all of a prompt but its last token goes into the cache, the prompts of a batch at once
    rest = [p[:-1] for p in prompts]
    if any(rest):
        ends = [0]
        for p in rest:
            ends.append(ends[-1] + len(p))
        model(torch.tensor(sum(rest, []), device="cuda"), _int32(ends), _int32([len(p) for p in rest]), cache)

    made = stood = 0
    rows = drafts + 1
    draft_starts, starts = (torch.arange(0, count * n + 1, n, dtype=torch.int32, device="cuda") for n in (1, rows))
    probabilities = torch.empty(count * rows, model.vocabulary, device="cuda")
    new, accepted = torch.empty(count * rows, dtype=torch.int32, device="cuda"), torch.empty(count, dtype=torch.int32, device="cuda")
    while min(len(t) - len(p) for t, p in zip(texts, prompts)) < steps:
        chunk = torch.empty(count, rows, dtype=torch.int32, device="cuda")
        chunk[:, 0] = _int32([t[-1] for t in texts])
        assert max(len(t) for t in texts) + drafts <= most      # (what the table has no page for would not be cached, and nobody told)
        cached = _int32([len(t) for t in texts])     # (with the last token, which the first draft appends)
        for i in range(drafts):
            logits = model(chunk[:, i].long(), draft_starts, cached + i, cache, blocks=1, most_new=1).float()
            p = torch.softmax(logits / max(temperature, 0.05), dim=1)
            probabilities.view(count, rows, -1)[:, i] = p
            chunk[:, i + 1] = torch.multinomial(p, 1, generator=gen)[:, 0].int()
        logits = model(chunk.view(-1).long(), starts, cached + drafts, cache, most_new=rows)
        uniforms = torch.rand(count * rows, generator=gen, device="cuda")
        H.hbp_verify_drafts(logits, chunk.view(-1), uniforms, starts, new, accepted, draft_probs=probabilities, temperature=heat)
        for text, tokens, n in zip(texts, new.view(count, rows).tolist(), accepted.tolist()):
            text += tokens[:n + 1]
            stood += n
        made += count * drafts
    return texts, stood, made


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("width", 256), ("blocks", 3), ("vocabulary", 2000), ("texts", 4), ("tokens", 40), ("drafts", 4), ("temperature", 0.8)):
        ap.add_argument("--" + name, type=type(default), default=default)
    a = ap.parse_args()
    model = Model(a.width, a.blocks, a.vocabulary)
    prompts = [[(7 * i + 3 * k) % a.vocabulary for k in range(5 + 9 * i)] for i in range(a.texts)]
    texts, stood, made = decode(model, prompts, a.tokens, a.drafts, a.temperature)
    for prompt, text in zip(prompts, texts):
        print(f"{len(prompt):4d} tokens, then " + " ".join(str(t) for t in text[len(prompt):len(prompt) + a.tokens]))
    print(f"{stood} of {made} drafted tokens stood")


if __name__ == "__main__":
    main()
