"""Verification of drafted tokens against the formula in 64 bits: whole numbers, equal to the last one."""
import ctypes

import numpy as np
import pytest

import paper_2504_08860_amd as H
from test_operators_q4 import TYPES, dtype

INF, NAN = float("inf"), float("nan")


def verify(logits, ids, uniforms, starts, temperature=None, draft_probs=None):
    """numpy, 64 bits: (new tokens, -2 in rows of no sequence; accepted)"""
    new, accepted = np.full(len(logits), -2), []
    for s, (a, b) in enumerate(zip(starts, starts[1:])):
        if not 0 <= a < b <= len(logits):
            accepted.append(0)
            continue
        heat = 1.0 if temperature is None else float(temperature[s])
        row, token, v = a, -1, logits.shape[1]
        while True:
            z = logits[row]
            top = z.max()
            good = np.isfinite(top) and not np.isnan(z).any() and heat >= 0
            if not good:
                p = np.full(v, NAN)
            elif heat == 0:
                p = (np.arange(v) == int(np.argmax(z))).astype(float)
            else:
                p = np.where(z == -INF, 0.0, np.exp((np.where(z == -INF, top, z) - top) / heat))
                p /= p.sum()
            if row == b - 1:
                w = p
                break
            d = int(ids[row + 1])
            q = (np.arange(v) == d).astype(float) if draft_probs is None else draft_probs[row]
            if 0 <= d < v and uniforms[row] * q[d] < p[d]:
                row += 1
                continue
            w = np.maximum(p - q, 0.0)
            if not w.sum() > 0:
                w = p
            break
        if w.sum() > 0:
            total = np.cumsum(w)
            over = np.flatnonzero((total > uniforms[b - 1] * total[-1]) & (w > 0))
            token = int(over[0] if len(over) else np.flatnonzero(w > 0)[-1])
        new[a:row] = ids[a + 1:row + 1]
        new[row], new[row + 1:b] = token, -1
        accepted.append(row - a)
    return new, np.array(accepted)


class Case:
    def __init__(self, counts, vocabulary, name, probabilities=True, heats=(1.0,), seed=0, behind=0, apart=0, wide_ids=False, spread=2.0):
        import torch
        rng = np.random.default_rng(seed)
        self.starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        n = int(self.starts[-1]) + behind
        z = rng.standard_normal((n, vocabulary)) * spread
        z[np.arange(n)[:, None], rng.integers(0, vocabulary, (n, 4))] += 6
        self.logits = torch.from_numpy(z.astype(np.float32)).to(dtype(name))
        self.temperature = None if heats is None else rng.choice(np.array(heats, np.float32), len(counts))
        row_heat = np.maximum(0.2, np.ones(len(counts)) if heats is None else self.temperature).repeat(counts)
        row_heat = np.concatenate([row_heat, np.ones(behind)])
        y = (z + 0.5 * rng.standard_normal(z.shape)) / row_heat[:, None]
        q = np.exp(y - y.max(1, keepdims=True)) if n else y
        q = (q / q.sum(1, keepdims=True)).astype(np.float32) if n else q.astype(np.float32)
        drawn = np.array([np.searchsorted(np.cumsum(r.astype(np.float64)), rng.random() * r.astype(np.float64).sum(), side="right") for r in q], np.int64).clip(0, vocabulary - 1)
        self.ids = np.concatenate([[0], drawn[:-1]]) if n else drawn
        self.q = q if probabilities else None
        self.uniforms = rng.random(n, dtype=np.float32)
        self.apart, self.wide_ids = apart, wide_ids

    def run(self, **how):
        import torch
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731

        def spaced(x):
            if not self.apart:
                return x.cuda()
            wide = torch.full((x.shape[0], x.shape[1] + 2 * self.apart), NAN, dtype=x.dtype, device="cuda")
            wide[:, self.apart:self.apart + x.shape[1]] = x.cuda()
            return wide[:, self.apart:self.apart + x.shape[1]]
        new = torch.full((len(self.ids),), -2, dtype=torch.int32, device="cuda")
        accepted = torch.full((len(self.starts) - 1,), 77, dtype=torch.int32, device="cuda")
        self.args = dict(logits=spaced(self.logits), tokens=t(self.ids.astype(np.int64 if self.wide_ids else np.int32)), uniforms=t(self.uniforms), starts=t(self.starts),
                         new_tokens=new, accepted=accepted, draft_probs=None if self.q is None else spaced(torch.from_numpy(self.q)),
                         temperature=None if self.temperature is None else t(self.temperature)) | how
        if "stream" in how:
            torch.cuda.synchronize()   # (the other stream waits for what was made on this one, and this one for it)
        H.hbp_verify_drafts(**self.args)
        if "stream" in how:
            how["stream"].synchronize()
        return new.cpu().numpy(), accepted.cpu().numpy()

    def want(self):
        return verify(self.logits.double().numpy(), self.ids, self.uniforms.astype(np.float64), self.starts, None if self.temperature is None else self.temperature.astype(np.float64),
                      None if self.q is None else self.q.astype(np.float64))

    def check(self, what=""):
        (new, accepted), (want_new, want_accepted) = self.run(), self.want()
        assert np.array_equal(accepted, want_accepted), f"{what}: {accepted.tolist()} and not {want_accepted.tolist()}"
        assert np.array_equal(new, want_new), f"{what}: rows {np.flatnonzero(new != want_new)[:10].tolist()}"
        return new, accepted


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("probabilities", [True, False])
def test_drafts(name, probabilities):
    some = 0
    for k, (counts, v) in enumerate([([1], 1), ([2, 1], 2), ([5], 7), ([3, 0, 1, 9, 0], 100), ([4] * 30, 1000), ([1, 2, 3, 4, 5, 6], 4096), ([6, 1, 3], 4097), ([2, 3], 9001), ([5, 4], 50_001),
                                     ([3], 300_007), ([17, 33], 333)]):
        for heats in (None, (0.0, 0.7, 1.0, 1.3), (0.0,)):
            print(f"[verify] {name} {counts} x {v} heats {heats}", flush=True)
            c = Case(counts, v, name, probabilities, heats, seed=k, behind=k % 3, apart=k % 2 * 3, wide_ids=k % 2 == 1)
            some += c.check(f"{counts} x {v}")[1].sum()
    assert some > 20     # (drafts stand and fall)


@pytest.mark.gpu
@pytest.mark.parametrize("probabilities", [True, False])
def test_draws_everywhere(probabilities):
    """The drawn place at the beginning, at the end, and from one token to the next; the same drafts, one place of many in each sequence."""
    v, n = 700, 400
    c = Case([2] * n, v, "f32", probabilities, None, seed=5)
    c.logits[:] = c.logits[:2].repeat(n, 1)
    c.ids[:] = np.tile([0, int(c.logits[0].argmin())], n)      # (an unlikely one)
    if probabilities:
        c.q[:] = np.tile(c.q[:2], (n, 1))
        c.q[0::2, c.ids[1]] += np.float32(0.01)
    c.uniforms[0::2] = 0.999
    c.uniforms[1::2] = np.linspace(0, 1, n, endpoint=False, dtype=np.float32)
    c.uniforms[-1] = np.float32(1 - 2.0 ** -24)
    new, accepted = c.check()
    assert accepted.sum() == 0 and len(set(new[0::2].tolist())) > 20
    c.uniforms[0::2] = 0.0      # all stand: the draw is the last row's
    if not probabilities:
        assert c.check()[1].sum() == n
    c.uniforms[1::2] = 1.5      # (beyond what there is: the last token with a weight)
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("v", [50, 9001])
def test_rows_of_every_odd_kind(name, v):
    """Masked tokens, nothing left, NaN and infinities, ties, drafts that are no tokens, temperatures that are none, probabilities that leave nothing."""
    for probabilities in (True, False):
        for where in (0, 1, 2):      # the row it happens in: drafts' rows and the last one
            for kind in range(13):
                c = Case([3] * 4, v, name, probabilities, (0.0, 1.0, 0.5), seed=kind, apart=1)
                c.uniforms[0::3], c.uniforms[1::3] = 0.0, 0.0 if kind % 2 else 0.4
                rows = slice(where, None, 3)
                z = c.logits[rows]
                if kind == 0:
                    z[:, ::2] = -INF
                elif kind == 1:
                    z[:] = -INF
                elif kind == 2:
                    z[:, v // 3] = NAN
                elif kind == 3:
                    z[:, v - 1] = INF
                elif kind == 4:
                    z[:] = 1.0
                elif kind == 5:
                    z[:, 5:] = -INF
                elif kind == 6:
                    z[:], z[:, v - 2] = -INF, -3.0
                elif kind == 7:
                    c.ids[rows] = [-1, v, v + 5, -2 ** 31]
                elif kind == 8:
                    c.temperature[:] = [-1.0, NAN, INF, 1e-38]
                elif kind == 9 and probabilities:
                    c.q[rows] = 2.0     # (nothing is left of p - q)
                elif kind == 10 and probabilities:
                    c.q[rows, ::2] = NAN
                elif kind == 11:
                    z *= 50
                elif kind == 12:
                    z[:], z[:, 3], z[:, v - 1] = float(np.float16(-60000)), 2.0, 2.0
                c.logits[rows] = z
                print(f"[verify odd] {name} {v} probabilities {probabilities} row {where} kind {kind}", flush=True)
                c.check(f"kind {kind} row {where}")


@pytest.mark.gpu
def test_long_rows_and_many():
    """Vocabularies beyond what one turn of 64 parts holds, rows further apart than 32 bits count, more sequences than a launch's grid has."""
    import torch
    c = Case([3, 2], 400_003, "bf16", True, (0.8,), seed=2)
    c.check("400003 tokens")
    v, n = 64, 70_001
    rng = np.random.default_rng(1)
    c = Case([2] * n, v, "f16", False, None, seed=3)
    c.check("70001 sequences")
    c = Case([2, 2], 1000, "f32", True, None, seed=4)
    want = c.want()
    far = torch.empty((3 << 30) + 5000, dtype=torch.bfloat16, device="cuda")
    z = far.as_strided((4, 1000), ((1 << 30) + 7, 1))
    z.copy_(c.logits)
    c.logits = z.cpu()
    want = c.want()
    new, accepted = c.run(logits=z)
    assert np.array_equal(new, want[0]) and np.array_equal(accepted, want[1]) and rng is not None


@pytest.mark.gpu
def test_streams_and_graphs():
    import torch
    c = Case([4] * 20, 20_000, "bf16", True, (0.0, 0.9, 1.0), seed=6)
    want = c.check()
    side = torch.cuda.Stream()
    new, accepted = c.run(stream=side)
    assert np.array_equal(new, want[0]) and np.array_equal(accepted, want[1])
    a = dict(c.args)
    a.pop("stream")
    H.hbp_verify_drafts(**a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        H.hbp_verify_drafts(**a)
    for k in range(3):
        a["uniforms"].uniform_()
        a["logits"].normal_(0, 3)
        H.hbp_verify_drafts(**a)
        eager = a["new_tokens"].clone(), a["accepted"].clone()
        a["new_tokens"].fill_(-5), a["accepted"].fill_(-5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a["new_tokens"], eager[0]) and torch.equal(a["accepted"], eager[1])


@pytest.mark.gpu
def test_shares_of_what_is_drawn():
    """Whatever the drafts are drawn from, the first new token of a sequence has the target's probabilities: 200000 sequences, counts within five standard deviations."""
    import torch
    n, v = 200_000, 12
    g = torch.Generator(device="cuda").manual_seed(0)
    z = torch.randn(1, v, generator=g, device="cuda") * 1.5
    q = torch.softmax(torch.randn(1, v, generator=g, device="cuda"), 1)
    drafts = torch.multinomial(q[0], n, replacement=True, generator=g).int()
    ids = torch.zeros(2 * n, dtype=torch.int32, device="cuda")
    ids[1::2] = drafts
    new, accepted = torch.empty_like(ids), torch.empty(n, dtype=torch.int32, device="cuda")
    H.hbp_verify_drafts(z.repeat(2 * n, 1), ids, torch.rand(2 * n, generator=g, device="cuda"), torch.arange(0, 2 * n + 1, 2, dtype=torch.int32, device="cuda"), new, accepted,
                        draft_probs=q.repeat(2 * n, 1))
    p = torch.softmax(z[0].double(), 0)
    counts = torch.bincount(new[0::2].long(), minlength=v).double()
    assert ((counts - n * p).abs() <= 5 * (n * p * (1 - p)).sqrt()).all()
    share = torch.minimum(p, q[0].double()).sum()
    assert (accepted.double().mean() - share).abs() <= 5 * (share * (1 - share) / n).sqrt()


def test_what_the_library_refuses():
    L = H.lib()
    need = ctypes.c_size_t()
    assert L.hbp_verify_drafts_workspace(4, 100, 2, need) == 0 and need.value > 0
    enough = need.value

    def call(type=0, z=4096, ldz=100, rows=4, v=100, ids=4096, idb=8, u=4096, starts=4096, n=2, heat=4096, q=4096, ldp=100, new=4096, acc=4096, ws=4096, size=enough):
        return L.hbp_verify_drafts(type, z, ldz, rows, v, ids, idb, u, starts, n, heat, q, ldp, new, acc, ws, size, None)
    for bad in (dict(type=3), dict(type=-1), dict(z=None), dict(z=4098), dict(ldz=99), dict(rows=-1), dict(v=0), dict(ids=None), dict(ids=4100), dict(idb=2), dict(u=None), dict(u=4097),
                dict(starts=None), dict(starts=4098), dict(n=-1), dict(heat=4097), dict(q=4098), dict(ldp=99), dict(new=None), dict(new=4097), dict(acc=None), dict(acc=4098),
                dict(ws=None), dict(ws=4100), dict(size=enough - 1)):
        assert call(**bad) == -1, bad
    for large in (dict(rows=(1 << 30) + 1), dict(v=(1 << 30) + 1), dict(n=(1 << 24) + 1)):
        assert call(**large) == -4, large
    assert call(n=0) == 0
    assert L.hbp_verify_drafts_workspace(4, 100, 2, None) == -1 and L.hbp_verify_drafts_workspace(0, 100, 2, need) == 0 and need.value == 0


@pytest.mark.gpu
def test_what_the_binding_refuses():
    import torch
    c = Case([2, 3], 60, "f16", True, (1.0,))
    c.run()
    good = c.args
    t = good
    for change in (dict(logits=t["logits"][0]), dict(logits=t["logits"].double()), dict(logits=t["logits"].t()), dict(logits=t["logits"].cpu()), dict(tokens=t["tokens"][:3]),
                   dict(tokens=t["tokens"].short()), dict(tokens=None), dict(uniforms=t["uniforms"].double()), dict(uniforms=t["uniforms"][:2]), dict(starts=t["starts"][:2]),
                   dict(starts=t["starts"].long()), dict(new_tokens=t["new_tokens"].long()), dict(new_tokens=t["new_tokens"][:4]), dict(accepted=t["accepted"][0]),
                   dict(accepted=t["accepted"].long()), dict(draft_probs=t["draft_probs"].half()), dict(draft_probs=t["draft_probs"][:, :5]), dict(temperature=t["temperature"].double()),
                   dict(temperature=t["temperature"][:1])):
        with pytest.raises(AssertionError):
            H.hbp_verify_drafts(**good | change)
    e = lambda *shape, kind=torch.int32: torch.empty(*shape, dtype=kind, device="cuda")  # noqa: E731
    accepted = torch.full((2,), 9, dtype=torch.int32, device="cuda")
    H.hbp_verify_drafts(e(0, 60, kind=torch.float32), e(0), e(0, kind=torch.float32), torch.zeros(3, dtype=torch.int32, device="cuda"), e(0), accepted)
    assert (accepted == 0).all()      # (no rows)
