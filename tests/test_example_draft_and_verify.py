"""The example's model over its paged cache against the same model in 64 bits without a cache; decoding with drafts against decoding token by token."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("draft_and_verify", os.path.join(ROOT, "examples", "draft_and_verify.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def reference(m, tokens, blocks=None):
    """Logits behind each token of one text, in 64 bits, from the values that the packed matrices stand for."""
    import torch
    rms = lambda v: v / (v.square().mean(-1, keepdim=True) + m.eps).sqrt()  # noqa: E731
    mm = lambda x, q: x @ q.values().double().t().contiguous()  # noqa: E731
    n, dim = len(tokens), m.head_dim
    h = m.embedding[tokens].double()
    x = rms(h) * m.w_in.double()
    angle = torch.arange(n, device="cuda").double()[:, None, None] * m.frequencies.double()
    cos, sin = angle.cos(), angle.sin()

    def turn(v):
        a, b = v[..., :dim // 2], v[..., dim // 2:]
        return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    for k in range(len(m.qkv) if blocks is None else blocks):
        q, key, value = (p.reshape(n, -1, dim) for p in mm(x, m.qkv[k]).split([m.heads * dim, m.kv_heads * dim, m.kv_heads * dim], 1))
        q, key = turn(q), turn(key)
        out = torch.empty_like(q)
        for head in range(m.heads):
            of = head // (m.heads // m.kv_heads)
            s = 30.0 * torch.tanh(q[:, head] @ key[:, of].t().contiguous() * dim ** -0.5 / 30.0)
            s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -float("inf"))
            out[:, head] = torch.softmax(s, 1) @ value[:, of]
        h = h + m.scales[k] * rms(mm(out.reshape(n, -1), m.out[k])) * m.norms[k][0].double()
        x = rms(h) * m.norms[k][1].double()
        h = h + m.scales[k] * rms(mm(torch.nn.functional.silu(mm(x, m.up[k])), m.down[k])) * m.norms[k][2].double()
        x = rms(h) * m.norms[k][3].double()
    return mm(x, m.head)


def test_logits_of_prompts_chunks_and_single_tokens(example):
    """Texts go in as prompts, then in chunks, then token by token, beside each other: each token's logits are those of the text without a cache."""
    import torch
    m = example.Model(192, 2, 501, heads=6, kv_heads=2, seed=2)
    g = torch.Generator().manual_seed(3)
    texts = [torch.randint(0, 501, (n,), generator=g) for n in (70, 33, 100)]
    cache, done = m.cache(3, 110), [0, 0, 0]
    wants = [reference(m, t.cuda()) for t in texts]
    for new in ((60, 1, 50), (0, 20, 3), (1, 1, 1), (7, 0, 40), (2, 11, 6)):
        starts = [0, new[0], new[0] + new[1], sum(new)]
        tokens = torch.cat([t[d:d + n] for t, d, n in zip(texts, done, new)]).cuda()
        done = [d + n for d, n in zip(done, new)]
        logits = m(tokens, example._int32(starts), example._int32(done), cache, most_new=max(new))
        for s in range(3):
            want = wants[s][done[s] - new[s]:done[s]]
            got = logits[starts[s]:starts[s + 1]].double()
            assert torch.allclose(got, want, atol=2e-4, rtol=0), (new, s, (got - want).abs().max().item())   # (logits are of size 3: some hundred roundings of fp32 through two blocks)


def test_greedy_decoding_with_drafts_is_greedy_decoding(example):
    import torch
    m = example.Model(192, 3, 501, heads=6, kv_heads=3, seed=5)
    prompts = [[5, 9, 11], [400], list(range(40))]
    texts, stood, made = example.decode(m, prompts, 12, drafts=3)
    assert 0 < stood < made
    for prompt, text in zip(prompts, texts):
        assert text[:len(prompt)] == prompt and len(text) >= len(prompt) + 12
        z = reference(m, torch.tensor(text, device="cuda"))
        for at in range(len(prompt), len(text)):
            best = z[at - 1].max().item()
            assert z[at - 1, text[at]].item() >= best - 1e-3      # (the best one, or as good as it in fp32)


def test_16_bit_models_run(example):
    import torch
    for dtype in (torch.float16, torch.bfloat16):
        m = example.Model(256, 2, 300, dtype=dtype, seed=7)
        texts, stood, made = example.decode(m, [[1, 2, 3], list(range(30))], 10, drafts=4, temperature=0.8)
        assert all(0 <= t < 300 for text in texts for t in text) and 0 <= stood <= made


def test_one_text_whose_drafts_all_stand_beside_one_whose_never_do(example):
    """The first text gets drafts + 1 tokens a round and the second one 1: the table has pages for all of them."""
    import torch

    class Steered(example.Model):
        def cache(self, texts, most, **how):
            made = super().cache(texts, most, **how)
            self.room = made[1].shape[1] * made[0][0][0].shape[2]
            return made

        def __call__(self, tokens, starts, lengths, cache, blocks=None, most_new=None):
            logits = super().__call__(tokens, starts, lengths, cache, blocks, most_new)
            assert int(lengths.max()) <= self.room, f"{lengths.tolist()} positions in a table for {self.room}"
            wanted = torch.zeros(len(tokens), dtype=torch.long, device="cuda") + 7
            wanted[int(starts[1]):] = 8 if blocks else 9      # (drafts of the second text are 8, and the whole model wants 9)
            return torch.full_like(logits, -20.0).scatter_(1, wanted[:, None], 20.0)
    m = Steered(192, 2, 50, heads=6, kv_heads=2, seed=1)
    for steps, drafts in ((12, 3), (5, 7), (1, 1)):
        texts, stood, made = example.decode(m, [[1, 2, 3], [4] * 9], steps, drafts=drafts)
        assert texts[0][3:] == [7] * (steps * (drafts + 1)) and texts[1][9:] == [9] * steps and 2 * stood == made == 2 * steps * drafts
