"""The example's model, token by token, against the same model in 64 bits; its tuning step against differences."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture()
def model():
    spec = importlib.util.spec_from_file_location("decode_and_tune", os.path.join(ROOT, "examples", "decode_and_tune.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    m = example.Model(200, 333, 1501, seed=3)
    yield m
    m.free()


def rms(v, eps):
    return v / (v.square().mean(-1, keepdim=True) + eps).sqrt()


def log_probabilities(m, tokens, gate=None):
    """Of all tokens behind each of `tokens`, in 64 bits, from the values that the packed matrices stand for."""
    import torch
    d = lambda t: t.double()  # noqa: E731
    h = d(m.embedding[tokens])
    x = rms(h, m.eps) * d(m.w_in)
    for k in range(len(m.up)):
        y = torch.nn.functional.silu(x @ d(m.up[k].values()).t().contiguous()) @ d(m.down[k].kept).t().contiguous()
        g = d(m.gate[k]) if gate is None or k + 1 < len(m.up) else gate
        h = h + m.scale * g * rms(y, m.eps) * d(m.w_post[k])
        x = rms(h, m.eps) * d(m.w_pre[k])
    return torch.log_softmax(x @ d(m.head.values()).t().contiguous(), -1)


def test_decoding(model):
    token = 7
    for out in model.decode(token, 6):
        lp = log_probabilities(model, [token])[0]
        best, ids = lp.sort(descending=True, stable=True)
        token, logp, entropy, got_ids, got_best = out
        assert got_ids == ids[:5].tolist() and token == got_ids[0]     # (apart by far more than fp32 is off)
        assert abs(logp - best[0].item()) < 1e-4 and abs(entropy + (lp.exp() * lp).sum().item()) < 1e-4
        assert max(abs(a - b) for a, b in zip(got_best, best[:5].tolist())) < 1e-4


def test_tuning(model):
    import torch
    tokens, wanted, bonus = list(range(10)), list(range(100, 110)), 0.01
    gate = model.gate[-1].double()

    def loss(g):
        lp = log_probabilities(model, tokens, g)
        return -(lp[torch.arange(10), wanted] - bonus * (lp.exp() * lp).sum(1)).mean()
    direction = torch.randn(200, generator=torch.Generator().manual_seed(1)).double().cuda()
    difference = ((loss(gate + 1e-5 * direction) - loss(gate - 1e-5 * direction)) / 2e-5).item()
    first = model.tune(tokens, wanted, bonus=bonus)
    along = (model.gradients["gate"].double() * direction)
    assert abs(along.sum().item() - difference) <= 1e-4 * along.abs().sum().item()
    for _ in range(5):
        last = model.tune(tokens, wanted, bonus=bonus)
    assert last > first
