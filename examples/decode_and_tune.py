#!/usr/bin/env python3
"""A small language model out of this library's products, decoding tokens one by one and tuning what can be tuned beside frozen weights.

A block is: a dense matrix in 4 bits (hbp_q4_mv), an activation, a pruned matrix in the sparse format (hbp_spmv), and between two blocks
the residual sum with a gate and the norms on both sides of it (hbp_residual_norms).  The output matrix is in 4 bits, too, and what is read off
the logits are log probabilities of the tokens, their entropy and the best alternatives (hbp_token_logprobs).

Tuning changes the last block's gate and norm weights so that given tokens become more likely: the logits' gradient
(hbp_token_logprobs_backward) goes through the frozen output matrix (hbp_q4_mv_t) and the norms (hbp_residual_norms_backward).

    python examples/decode_and_tune.py [--width 512] [--inner 1536] [--vocabulary 5000] [--tokens 16]
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

    def __init__(self, w, group=64):
        codes, scales = H.hbp_q4_shapes(*w.shape, group)
        self.shape, self.group = tuple(w.shape), group
        self.codes = torch.empty(codes, dtype=torch.uint8, device="cuda")
        self.scales = torch.empty(scales, dtype=torch.float16, device="cuda")
        H.hbp_q4_pack(w, self.codes, self.scales, group=group)

    def __call__(self, x):
        y = x.new_empty(*x.shape[:-1], self.shape[0])
        H.hbp_q4_mv(self.codes, self.scales, x, y, group=self.group)
        return y

    def backward(self, dy):
        dx = dy.new_empty(*dy.shape[:-1], self.shape[1])
        H.hbp_q4_mv_t(self.codes, self.scales, dy, dx, group=self.group)
        return dx

    def values(self):
        return H.hbp_q4_unpack(self.codes, self.scales, self.shape[1], group=self.group)


class Pruned:
    """A matrix of which the smallest nine tenths are gone."""

    def __init__(self, w):
        keep = w.abs() >= w.abs().flatten().kthvalue(int(0.9 * w.numel())).values
        rows, cols = keep.nonzero(as_tuple=True)
        ptr = torch.zeros(w.shape[0] + 1, dtype=torch.int64, device="cuda")
        ptr[1:] = torch.cumsum(keep.sum(1), 0)
        self.shape, self.kept = tuple(w.shape), w * keep
        self.handle = H.hbp_build(ptr.int(), cols.int(), w[rows, cols].contiguous(), *w.shape)

    def __call__(self, x):
        y = x.new_empty(self.shape[0])
        H.hbp_spmv(self.handle, x, y)
        return y

    def free(self):
        H.hbp_free(self.handle)


class Model:
    def __init__(self, width, inner, vocabulary, blocks=2, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
        self.width, self.vocabulary, self.scale, self.eps = width, vocabulary, 0.5, 1e-6
        self.embedding = r(vocabulary, width)
        self.up = [Q4(r(inner, width) / width ** 0.5) for _ in range(blocks)]
        self.down = [Pruned(r(width, inner) / (0.1 * inner) ** 0.5) for _ in range(blocks)]
        self.w_post, self.w_pre, self.gate = ([1 + 0.1 * r(width) for _ in range(blocks)] for _ in range(3))
        self.w_in = 1 + 0.1 * r(width)
        self.head = Q4(r(vocabulary, width) * (2 / width ** 0.5))

    def hidden(self, token):
        """(h and the block's result before the last norms, what the output matrix sees) for one token"""
        h = self.embedding[token:token + 1].clone()
        y, x = torch.zeros_like(h), torch.empty_like(h)
        H.hbp_residual_norms(h, y, h, x, w_pre=self.w_in, eps=self.eps)   # (no block yet: the norm alone)
        before = None
        for k in range(len(self.up)):
            y = self.down[k](torch.nn.functional.silu(self.up[k](x[0])))[None]
            before = (h.clone(), y.clone())
            H.hbp_residual_norms(h, y, h, x, w_post=self.w_post[k], w_pre=self.w_pre[k], gate=self.gate[k], scale=self.scale, eps=self.eps)
        return before, x

    def decode(self, token, steps, top=5):
        """Greedy decoding: a list of (token, its log probability, entropy, the alternatives' ids and log probabilities)."""
        out = []
        logp, entropy = (torch.empty(1, device="cuda") for _ in range(2))
        ids, best = torch.empty(1, top, dtype=torch.int32, device="cuda"), torch.empty(1, top, device="cuda")
        for _ in range(steps):
            logits = self.head(self.hidden(token)[1])
            H.hbp_token_logprobs(logits, None, entropy=entropy, top_ids=ids, top_logp=best)
            token = int(ids[0, 0])
            H.hbp_token_logprobs(logits, ids[:, 0].contiguous(), logp)
            out.append((token, float(logp), float(entropy), ids[0].tolist(), best[0].tolist()))
        return out

    def tune(self, tokens, wanted, rate=0.5, bonus=0.01):
        """One step on the last block's gate and norm weights: raises the log probabilities of `wanted` behind `tokens`, with a bonus for entropy.
        Returns the mean log probability before the step."""
        n = len(tokens)
        states = [self.hidden(t)[0] for t in tokens]
        h, y = (torch.cat([s[i] for s in states]) for i in (0, 1))
        h_out, x, rstd = torch.empty_like(h), torch.empty_like(h), torch.empty(n, 2, device="cuda")
        last = dict(w_post=self.w_post[-1], w_pre=self.w_pre[-1], gate=self.gate[-1], scale=self.scale)
        H.hbp_residual_norms(h, y, h_out, x, rstd=rstd, eps=self.eps, **last)
        logits = self.head(x)
        wanted = torch.tensor(wanted, device="cuda")
        logp, entropy, lse = (torch.empty(n, device="cuda") for _ in range(3))
        H.hbp_token_logprobs(logits, wanted, logp, entropy, lse=lse)
        g_logp, g_entropy = torch.full((n,), -1.0 / n, device="cuda"), torch.full((n,), -bonus / n, device="cuda")   # of the loss -mean(logp + bonus H)
        H.hbp_token_logprobs_backward(logits, wanted, lse, entropy, g_logp, g_entropy, logits)                         # (in place)
        d_x = self.head.backward(logits)
        d_h, d_y = torch.empty_like(h), torch.empty_like(h)
        d = {k: torch.empty(self.width, device="cuda") for k in ("w_post", "w_pre", "gate")}
        H.hbp_residual_norms_backward(None, d_x, h, y, rstd, d_h, d_y, d_w_post=d["w_post"], d_w_pre=d["w_pre"], d_gate=d["gate"], **last)
        for parameter, key in ((self.w_post[-1], "w_post"), (self.w_pre[-1], "w_pre"), (self.gate[-1], "gate")):
            parameter -= rate * d[key]
        self.gradients = d
        return float(logp.mean())

    def free(self):
        for m in self.down:
            m.free()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("width", 512), ("inner", 1536), ("vocabulary", 5000), ("tokens", 16)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    model = Model(a.width, a.inner, a.vocabulary)
    try:
        for token, logp, entropy, ids, best in model.decode(1, a.tokens):
            print(f"token {token:6d}  log p {logp:8.4f}  entropy {entropy:7.4f}  alternatives " + " ".join(f"{i}:{p:.3f}" for i, p in zip(ids, best)))
        tokens, wanted = list(range(1, 25)), list(range(2, 26))
        for step in range(5):
            print(f"step {step}: mean log p of the wanted tokens {model.tune(tokens, wanted):.4f}")
    finally:
        model.free()


if __name__ == "__main__":
    main()
