"""Token log probabilities, entropies, alternatives and the logits' gradient, against numpy in 64 bits and against differences."""
import ctypes

import numpy as np
import pytest

import paper_2504_08860_amd as H
from test_operators_q4 import TINY, TYPES, UNIT, dtype

INF = float("inf")


def logits_of(n, vocabulary, name, seed, spread=3.0, masked=0.0):
    import torch
    rng = np.random.default_rng(seed)
    z = (spread * rng.standard_normal((n, vocabulary))).astype(np.float32)
    if masked:
        z[rng.random(z.shape) < masked] = -np.inf
    return torch.from_numpy(z).to(dtype(name))


def reference(z):
    """(log probabilities, p, entropy, lse) of rows in 64 bits; a row with nothing left: -inf, 0, 0, -inf"""
    m = z.max(1, keepdims=True)
    none = m == -np.inf
    with np.errstate(invalid="ignore", divide="ignore"):
        below = z - np.where(none, 0, m)      # (taken from the largest first: at 1e38 even 64 bits lose a logarithm next to it)
        log_sum = np.log(np.exp(below).sum(1, keepdims=True))
        lse = np.where(none, -np.inf, m + log_sum)
        lp = np.where(none, -np.inf, below - np.where(none, 0, log_sum))
        p = np.exp(lp)
        h = -np.where(p > 0, p * np.where(p > 0, lp, 0), 0).sum(1, keepdims=True)
    return lp, p, h, lse


def order(z, top):
    """NaN first, then descending, lowest index first among equals"""
    key = np.where(np.isnan(z), np.inf, z)
    return np.stack([np.lexsort((np.arange(z.shape[1]), -key[r], ~np.isnan(z[r])))[:top] for r in range(z.shape[0])])


def run(z, tokens, top=0, **more):
    import torch
    n = z.shape[0]
    f = lambda *s: torch.full(s, 99.0, device="cuda")  # noqa: E731
    out = {"logp": f(n), "entropy": f(n), "lse": f(n)}
    if tokens is None:
        out.pop("logp")
    if top:
        out |= {"top_ids": torch.full((n, top), -9, dtype=torch.int32, device="cuda"), "top_logp": f(n, top)}
    H.hbp_token_logprobs(z, tokens, **out, **more)
    torch.cuda.synchronize()
    return out


def near(got, want, size, what):
    """fp32: a logit, the row's largest one and the logarithm of a sum meet in a few roundings (8 allowed for) of the larger of them, and the
    sum's own error, 16 roundings of 1, is what it adds to its logarithm."""
    got = got.cpu().double().numpy()
    same = np.isinf(want) & (got == want)
    with np.errstate(invalid="ignore"):
        off = np.where(same, 0.0, np.abs(got - want))
    most = 2.0 ** -24 * (8 * size + 16)
    assert (off <= most).all(), f"{what}: off by {np.nanmax(off):.3g}"


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("masked", [0.0, 0.6])
def test_forward_and_backward(name, masked):
    import torch
    for k, (n, v, top) in enumerate(((1, 1, 1), (1, 5, 5), (3, 8, 3), (2, 63, 20), (5, 513, 1), (4, 4096, 64), (7, 4097, 7), (1, 50001, 20), (1, 8191, 0),
                                     (600, 1000, 3), (3, 20011, 50), (1, 140000, 33))):
        for id_type in (torch.int32, torch.int64):
            print(f"[logprobs] {n} x {v} top {top} {name} masked {masked} {id_type}", flush=True)
            z = logits_of(n, v, name, 100 * k + int(10 * masked), masked=masked)
            f = z.double().numpy()
            tokens = torch.from_numpy(np.random.default_rng(k).integers(0, v, n)).to(id_type)
            wide = torch.full((n, v + 5), float("nan"), dtype=z.dtype, device="cuda")
            wide[:, 2:2 + v] = z.cuda()
            zg = wide[:, 2:2 + v] if k % 2 else z.cuda()
            out = run(zg, tokens.cuda(), top)
            lp, p, h, lse = reference(f)
            size = np.abs(np.where(np.isfinite(f), f, 0)).max() + np.log(v) + 1
            near(out["lse"], lse[:, 0], size, "lse")
            near(out["logp"], np.take_along_axis(lp, tokens.long().numpy()[:, None], 1)[:, 0], size, "logp")
            near(out["entropy"], h[:, 0], size, "entropy")
            if top:
                ids = order(f, top)
                assert np.array_equal(out["top_ids"].cpu().numpy(), ids)
                near(out["top_logp"], np.take_along_axis(lp, ids, 1), size, "top_logp")
            u, w = torch.randn(n, generator=torch.Generator().manual_seed(k)), torch.randn(n, generator=torch.Generator().manual_seed(k + 1))
            d = torch.empty_strided(zg.shape, zg.stride(), dtype=z.dtype, device="cuda")
            H.hbp_token_logprobs_backward(zg, tokens.cuda(), out["lse"], out["entropy"], u.cuda(), w.cuda(), d)
            check_gradient(d, f, tokens.numpy(), u.numpy(), w.numpy(), name, size)


def gradient(f, tokens, u, w):
    lp, p, h, _ = reference(f)
    hit = (np.arange(f.shape[1]) == tokens[:, None]) * np.where(h == h, 1.0, 0.0)
    u, w = u.astype(np.float64)[:, None], w.astype(np.float64)[:, None]
    none = ~(f.max(1, keepdims=True) > -np.inf)
    with np.errstate(invalid="ignore"):
        d = u * (hit - p) - w * p * np.where(p > 0, np.where(p > 0, lp, 0) + h, 0)
    return np.where(none, 0.0, d), p, np.abs(u) + np.abs(w) * (np.where(p > 0, np.abs(np.where(p > 0, lp, 0)), 0) + h)


def check_gradient(d, f, tokens, u, w, name, size):
    """A probability is off by the roundings of z - lse (8 of `size`) relative to itself; the token's own term is u - u p."""
    want, p, weight = gradient(f, tokens, u, w)
    got = d.cpu().double().numpy()
    most = UNIT[name] * np.abs(want) * (1 + 1e-6) + 2.0 ** -24 * ((8 * size + 16) * p * (weight + np.abs(w)[:, None]) + 4 * np.abs(u)[:, None] * (p + (np.arange(f.shape[1]) == tokens[:, None])))
    off = np.abs(got - want)
    assert np.isfinite(got).all() and (off <= most + TINY[name]).all(), f"gradient: worst {np.max(off / (most + TINY[name])):.3g} times what is allowed"


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("v", [100, 9000])
def test_rows_of_every_odd_kind(name, v):
    """Nothing left, one left, the type's lowest value as a mask, all equal, NaN, +inf, ids that are no token or beyond the vocabulary."""
    import torch
    low = torch.finfo(dtype(name)).min
    z = logits_of(10, v, name, 4)
    z[0] = -INF                                      # nothing
    z[1] = -INF
    z[1, 57] = 2.0                                   # one
    z[2, ::2] = low                                  # a mask that is a number
    z[3] = 1.5                                       # all equal
    z[4, 60] = float("nan")
    z[5, 61] = INF
    z[6] = low                                       # nothing but the lowest value: a row like any other, all equal
    z[7, 3], z[7, 70] = -0.0, 0.0
    z[7, z[7] > 0] = -1.0
    tokens = torch.tensor([5, 57, 1, 3, 2, 61, 9, 3, -1, v], dtype=torch.int64)
    out = {k: t.cpu().double().numpy() for k, t in run(z.cuda(), tokens.cuda(), 4).items()}
    f = z.double().numpy()
    fine = [0, 1, 2, 3, 6, 7, 8, 9]
    lp, p, h, lse = reference(f[fine])
    size = np.abs(np.where(np.isfinite(lse), lse, 0)) + 30
    assert np.array_equal(np.isinf(out["lse"][fine]), np.isinf(lse[:, 0]))
    ids = order(f, 4)
    assert np.array_equal(out["top_ids"], ids)
    for r, row in enumerate(fine):
        if row == 0:
            assert out["lse"][0] == -INF and out["logp"][0] == -INF and out["entropy"][0] == 0 and (out["top_logp"][0] == -INF).all()
            continue
        assert abs(out["entropy"][row] - h[r, 0]) <= 2.0 ** -24 * (8 * np.log(v) + 16 + 8 * 30) + 1e-6
        assert abs(out["lse"][row] - lse[r, 0]) <= 2.0 ** -24 * 8 * size[r, 0]
        want = lp[r][ids[row]]
        finite = np.isfinite(want)
        assert np.array_equal(np.isfinite(out["top_logp"][row]), finite)
        near_ones = finite & (want > -1e3)
        assert (np.abs(out["top_logp"][row] - want)[near_ones] <= 2.0 ** -24 * 8 * 60).all()
    assert out["logp"][1] == 0 and out["entropy"][1] == 0
    assert abs(out["logp"][6] + np.log(v)) <= 1e-5 and abs(out["entropy"][6] - np.log(v)) <= 1e-5
    assert np.isnan(out["lse"][[4, 5]]).all() and np.isnan(out["logp"][[4, 5]]).all() and np.isnan(out["entropy"][[4, 5]]).all()
    assert out["logp"][8] == 0 and np.isnan(out["logp"][9])
    g = torch.full((10,), 0.5, device="cuda")
    o = run(z.cuda(), tokens.cuda())
    d = torch.empty_like(z, device="cuda")
    H.hbp_token_logprobs_backward(z.cuda(), tokens.cuda(), o["lse"], o["entropy"], g, g, d)
    d = d.cpu().double().numpy()
    assert not d[0].any() and np.isfinite(d[[0, 1, 2, 3, 6, 7, 8]]).all() and np.isnan(d[9]).all() and np.isnan(d[[4, 5]]).any(1).all()
    assert not d[2, ::2].any()
    want, p, _ = gradient(f[8:9], np.array([-1]), np.zeros(1), np.array([0.5]))     # no token: the entropy's part alone
    assert (np.abs(d[8] - want) <= (UNIT[name] + 1e-5) * (np.abs(want) + p) + TINY[name]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("v", [700, 30000])
def test_alternatives_in_the_worst_orders(v):
    """Ascending logits (every one is a new best), descending ones, few values with many ties, fewer unmasked tokens than alternatives."""
    import torch
    z = np.zeros((5, v), np.float32)
    z[0], z[1] = np.linspace(-5, 5, v), np.linspace(5, -5, v)
    z[2] = np.random.default_rng(1).integers(0, 3, v)
    z[3] = -np.inf
    z[3, [v - 1, 7, v // 2]] = [1, 1, 2]
    z[4] = -3.0
    for top in (1, 2, 31, 64):
        out = run(torch.from_numpy(z).cuda(), None, top)
        ids = order(z.astype(np.float64), top)
        assert np.array_equal(out["top_ids"].cpu().numpy(), ids)
        lp = reference(z.astype(np.float64))[0]
        near(out["top_logp"], np.take_along_axis(lp, ids, 1), 20.0, "top_logp")


@pytest.mark.gpu
def test_gradient_against_differences():
    """Of sum(u logp + w H) along random directions, by central differences of the 64-bit formula."""
    import torch
    n, v, step = 5, 301, 1e-5
    z = logits_of(n, v, "f32", 9, masked=0.3)
    z[:, 17] = 0.5
    f, tokens = z.double().numpy(), np.full(n, 17)
    rng = np.random.default_rng(2)
    u, w = rng.standard_normal(n).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    t = lambda a: torch.from_numpy(np.asarray(a)).cuda()  # noqa: E731
    out = run(z.cuda(), t(tokens))
    d = torch.empty_like(z, device="cuda")
    H.hbp_token_logprobs_backward(z.cuda(), t(tokens), out["lse"], out["entropy"], t(u), t(w), d)

    def loss(a):
        lp, _, h, _ = reference(a)
        return (u * lp[:, 17]).sum() + (w * h[:, 0]).sum()
    for _ in range(5):
        direction = rng.standard_normal(f.shape)
        difference = (loss(f + step * direction) - loss(f - step * direction)) / (2 * step)
        along = d.cpu().double().numpy() * direction
        assert abs(along.sum() - difference) <= 1e-5 * (np.abs(along).sum() + 1)


@pytest.mark.gpu
def test_in_place_missing_parts_streams_and_graph():
    import torch
    n, v = 70, 12345
    z = logits_of(n, v, "bf16", 21).cuda()
    tokens = torch.randint(0, v, (n,), device="cuda")
    first = run(z, tokens, 10)
    alone = torch.empty(n, device="cuda")
    H.hbp_token_logprobs(z, None, entropy=alone)
    assert torch.equal(alone, first["entropy"])
    H.hbp_token_logprobs(z, tokens, logp=alone)
    assert torch.equal(alone, first["logp"])
    u, w, zero = torch.randn(n, device="cuda"), torch.randn(n, device="cuda"), torch.zeros(n, device="cuda")
    one, two = torch.empty_like(z), torch.empty_like(z)
    for a, b in ((u, None), (None, w), (None, None)):
        H.hbp_token_logprobs_backward(z, tokens, first["lse"], first["entropy"], a, b, one)
        H.hbp_token_logprobs_backward(z, tokens, first["lse"], first["entropy"], zero if a is None else a, zero if b is None else b, two)
        assert torch.equal(one, two)
    H.hbp_token_logprobs_backward(z, tokens, first["lse"], first["entropy"], u, w, one)
    again = z.clone()
    H.hbp_token_logprobs_backward(again, tokens, first["lse"], first["entropy"], u, w, again)
    assert torch.equal(again, one)
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        side.wait_stream(torch.cuda.current_stream())
        there = run(z, tokens, 10, stream=stream)
        assert all(torch.equal(there[k], first[k]) for k in first)
    few = z[:1].clone()                      # a row in parts, joined by a second kernel
    out = run(few, tokens[:1], 10)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        H.hbp_token_logprobs(few, tokens[:1], **out)
        H.hbp_token_logprobs_backward(few, tokens[:1], out["lse"], out["entropy"], u[:1], w[:1], two[:1])
    for k in range(3):
        few.copy_(z[k:k + 1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(two[:1], torch.where(torch.isnan(two[:1]), two[:1], two[:1]))
        eager = run(few, tokens[:1], 10)
        assert all(torch.equal(out[key], eager[key]) for key in eager)
        H.hbp_token_logprobs_backward(few, tokens[:1], eager["lse"], eager["entropy"], u[:1], w[:1], one[:1])
        assert torch.equal(one[:1], two[:1])


@pytest.mark.gpu
def test_rows_further_apart_than_32_bits_count_and_many_rows():
    import torch
    apart, v = (1 << 32) + 24, 5000
    wide = torch.empty(apart + v, dtype=torch.bfloat16, device="cuda")
    far = wide.as_strided((2, v), (apart, 1))
    z = logits_of(2, v, "bf16", 31).cuda()
    far.copy_(z)
    tokens = torch.tensor([4, 4999], device="cuda")
    a, b = run(z, tokens, 5), run(far, tokens, 5)
    assert all(torch.equal(a[k], b[k]) for k in a)
    g, d, e = torch.ones(2, device="cuda"), torch.empty_like(z), torch.empty_like(z)
    H.hbp_token_logprobs_backward(far, tokens, a["lse"], a["entropy"], g, g, d)
    H.hbp_token_logprobs_backward(z, tokens, a["lse"], a["entropy"], g, g, far)
    e.copy_(far)
    assert torch.equal(d, e)
    n = 70_001                               # more rows than one launch takes
    z = torch.randn(n, 9, device="cuda")
    tokens = torch.randint(0, 9, (n,), device="cuda")
    out = run(z, tokens, 2)
    lp = torch.log_softmax(z.double(), 1)
    assert (out["logp"] - lp.gather(1, tokens[:, None])[:, 0]).abs().max() <= 2e-6
    assert torch.equal(out["top_ids"].long(), torch.sort(z, dim=1, descending=True, stable=True).indices[:, :2])
    d = torch.empty_like(z)
    g = torch.ones(n, device="cuda")
    H.hbp_token_logprobs_backward(z, tokens, out["lse"], out["entropy"], g, None, d)
    assert (d - (torch.nn.functional.one_hot(tokens, 9) - lp.exp())).abs().max() <= 2e-6


@pytest.mark.gpu
def test_no_rows_and_what_the_binding_refuses():
    import torch
    none = torch.empty(0, 50, device="cuda")
    f = torch.empty(0, device="cuda")
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    H.hbp_token_logprobs(none, ids, f, f, lse=f)
    H.hbp_token_logprobs_backward(none, ids, f, f, f, f, none)
    z, t, o = torch.zeros(2, 50, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(2, device="cuda")
    good = dict(logits=z, tokens=t, logp=o)
    i, p = torch.zeros(2, 5, dtype=torch.int32, device="cuda"), torch.zeros(2, 5, device="cuda")
    for change in (dict(logits=z.double()), dict(logits=z.cpu()), dict(logits=z[0]), dict(tokens=t[:1]), dict(tokens=t.short()), dict(logp=o[:1]),
                   dict(logp=o.half()), dict(top_ids=i), dict(top_ids=i.long(), top_logp=p), dict(top_ids=i, top_logp=p[:, :3]), dict(logits=z.t())):
        with pytest.raises(AssertionError):
            H.hbp_token_logprobs(**good | change)
    for change in (dict(tokens=None), dict(top_ids=torch.zeros(2, 51, dtype=torch.int32, device="cuda"), top_logp=torch.zeros(2, 51, device="cuda"))):
        with pytest.raises(H.HbpError) as e:
            H.hbp_token_logprobs(**good | change)
        assert e.value.status == -1


def test_what_the_library_refuses():
    L = H.lib()
    need = ctypes.c_size_t()
    ok = dict(type=0, z=4096, ldz=100, n=2, v=100, ids=4096, idb=8, logp=4096, ent=None, lse=None, top=0, ti=None, tp=None, ws=None, size=0)

    def call(**k):
        a = ok | k
        return L.hbp_token_logprobs(a["type"], a["z"], a["ldz"], a["n"], a["v"], a["ids"], a["idb"], a["logp"], a["ent"], a["lse"], a["top"], a["ti"], a["tp"],
                                    a["ws"], a["size"], None)
    for bad in (dict(type=3), dict(z=None), dict(z=4098), dict(ldz=99), dict(n=-1), dict(v=0), dict(idb=2), dict(ids=4100), dict(ids=None), dict(logp=4098), dict(top=-1),
                dict(top=65), dict(top=3), dict(top=3, ti=4096), dict(ent=4097), dict(lse=4099)):
        assert call(**bad) == -1, bad
    assert call(n=0) == 0 and call(v=1 << 31, ldz=1 << 31) == -4
    assert L.hbp_token_logprobs_workspace(0, 1, 100000, 5, need) == 0 and need.value > 0
    for ws, size in ((4096, need.value - 1), (None, need.value), (4100, need.value)):
        assert call(n=1, v=100000, ldz=100000, top=5, ti=4096, tp=4096, ws=ws, size=size) == -1
    assert L.hbp_token_logprobs_workspace(0, 1, 100, 101, need) == -1 and L.hbp_token_logprobs_workspace(0, 1, 100, 5, None) == -1
    back = lambda type=0, z=4096, ldz=100, ids=4096, idb=8, lse=4096, ent=4096, g=4096, w=4096, d=4096, ldd=100, n=2: L.hbp_token_logprobs_backward(  # noqa: E731
        type, z, ldz, n, 100, ids, idb, lse, ent, g, w, d, ldd, None)
    for bad in (dict(type=9), dict(z=None), dict(ldz=1), dict(ids=None), dict(idb=1), dict(lse=None), dict(ent=None), dict(d=None), dict(ldd=99), dict(d=4097), dict(g=4097)):
        assert back(**bad) == -1, bad
    assert back(n=0) == 0


@pytest.mark.gpu
def test_alternatives_of_other_dimensions_are_refused():
    import torch
    z, t, o = torch.zeros(2, 50, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(2, device="cuda")
    for shape in ((), (2,), (2, 5, 1)):
        with pytest.raises(AssertionError):
            H.hbp_token_logprobs(z, t, o, top_ids=torch.zeros(shape, dtype=torch.int32, device="cuda"), top_logp=torch.zeros(shape, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("v", [100, 9000, 40001])
def test_gradient_of_logits_far_from_zero(name, v):
    """Logits around a number that lse, in 32 bits, holds only roughly or not at all: a probability is that of the difference to the largest one, whose roundings are
    relative to itself and to ln v (check_gradient's `size`, not that of the logits), and a row's gradient for its token's logit adds up to zero."""
    import torch
    low = float(torch.finfo(dtype(name)).min)
    for k, at in enumerate([20.0, 30.0, 200.0, -1000.0, 1e4, -6e4] + ([] if name == "f16" else [1e6, 1e8, -1e8, 3e38]) + [low]):
        for masked in (0.0, 0.4):
            print(f"[logprobs far] {v} {name} around {at} masked {masked}", flush=True)
            z = logits_of(4, v, "f32", 50 + k)
            z = (z + at if at != low else torch.full_like(z, low)).to(dtype(name))
            gone = torch.from_numpy(np.random.default_rng(k).random((4, v)) < masked)
            gone[:, 7] = False
            z[gone] = -INF
            f, tokens = z.double().numpy(), torch.tensor([7, 3, -1, v - 1])
            wide = torch.full((4, v + 5), float("nan"), dtype=z.dtype, device="cuda")
            wide[:, 2:2 + v] = z.cuda()
            zg = wide[:, 2:2 + v] if k % 2 else z.cuda()
            out = run(zg, tokens.cuda())
            u, w = (torch.randn(4, generator=torch.Generator().manual_seed(k + i)) for i in (0, 1))
            u[2] = 0.0                                 # (no token: nothing comes from there)
            d = torch.empty_like(zg)
            H.hbp_token_logprobs_backward(zg, tokens.cuda(), out["lse"], out["entropy"], u.cuda(), w.cuda(), d)
            check_gradient(d, f, tokens.numpy(), u.numpy(), w.numpy(), name, np.log(v) + 4)
            if name == "f32":
                only = torch.empty_like(zg)
                H.hbp_token_logprobs_backward(zg, tokens.cuda(), out["lse"], out["entropy"], u.cuda(), None, only)
                assert (only.double().sum(1).abs().cpu() <= 2.0 ** -24 * (8 * (np.log(v) + 4) + 16 + 4) * u.abs().double()).all()
            H.hbp_token_logprobs_backward(zg, tokens.cuda(), out["lse"], out["entropy"], u.cuda(), w.cuda(), zg)      # in place
            assert torch.equal(zg, d)


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
def test_rows_far_from_zero_among_others(name):
    """Every third row around 10000, more rows than those that workgroups of another size take: gradients as of each row alone, in place, too."""
    import torch
    for n, v in ((400, 3000), (257, 20011)):
        print(f"[logprobs far] {n} x {v} {name} among others", flush=True)
        z = logits_of(n, v, "f32", n)
        z[::3] += 1e4
        z = z.to(dtype(name))
        tokens = torch.from_numpy(np.random.default_rng(n).integers(0, v, n))
        out = run(z.cuda(), tokens.cuda())
        u, w = (torch.randn(n, generator=torch.Generator().manual_seed(i)) for i in (1, 2))
        d, zg = torch.empty_like(z, device="cuda"), z.cuda()
        H.hbp_token_logprobs_backward(zg, tokens.cuda(), out["lse"], out["entropy"], u.cuda(), w.cuda(), d)
        check_gradient(d, z.double().numpy(), tokens.numpy(), u.numpy(), w.numpy(), name, np.log(v) + 4)
        H.hbp_token_logprobs_backward(zg, tokens.cuda(), out["lse"], out["entropy"], u.cuda(), w.cuda(), zg)
        assert torch.equal(zg, d)
