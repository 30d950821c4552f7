"""Residual norms, forward and backward, against numpy in 64 bits and against differences."""
import ctypes

import numpy as np
import pytest

import paper_2504_08860_amd as H
from test_operators_q4 import TINY, TYPES, UNIT, dtype, some_x

EPS = 1e-5
GATES = ["none", "channel", "token", "full"]


def inputs(tokens, width, name, gate, seed, weights=True):
    import torch
    t = {"h": some_x(tokens, width, name, seed), "y": some_x(tokens, width, name, seed + 1) * 3}
    t["w_post"], t["w_pre"] = ((1 + 0.2 * some_x(1, width, name, seed + k)[0]) if weights else None for k in (2, 3))
    shape = {"none": None, "channel": (1, width), "token": (tokens, 1), "full": (tokens, width)}[gate]
    t["gate"] = None if shape is None else some_x(*shape, name, seed + 4)
    if gate == "channel":
        t["gate"] = t["gate"][0]
    t["d_h_out"], t["d_x_out"] = some_x(tokens, width, name, seed + 5), some_x(tokens, width, name, seed + 6)
    assert all(v is None or v.dtype == dtype(name) for v in t.values()) and torch.is_tensor(t["h"])
    return t


def forward(t, scale, eps):
    """numpy, 64 bits: outputs, and what the backward formulas use"""
    f = {k: None if v is None else np.asarray(v, np.float64) for k, v in t.items()}
    one = lambda v: 1.0 if v is None else v  # noqa: E731
    q1 = np.sqrt((f["y"] ** 2).mean(1, keepdims=True) + eps)
    n = f["y"] / q1 * one(f["w_post"])
    h2 = f["h"] + scale * one(f["gate"]) * n
    q2 = np.sqrt((h2 ** 2).mean(1, keepdims=True) + eps)
    return h2, h2 / q2 * one(f["w_pre"]), n, q1, q2


def backward(t, scale, eps, gate):
    f = {k: None if v is None else np.asarray(v, np.float64) for k, v in t.items()}
    one = lambda v: 1.0 if v is None else v  # noqa: E731
    h2, _, n, q1, q2 = forward(t, scale, eps)
    width = h2.shape[1]
    through = lambda g, v, q: (g - v / q * (g * v / q).sum(1, keepdims=True) / width) / q  # noqa: E731
    dh, dx = (np.zeros_like(h2) if f[k] is None else f[k] for k in ("d_h_out", "d_x_out"))
    e = dh + through(dx * one(f["w_pre"]), h2, q2)
    ge = scale * one(f["gate"]) * e
    out = {"d_h": e, "d_y": through(ge * one(f["w_post"]), f["y"], q1), "d_w_post": (ge * f["y"] / q1).sum(0), "d_w_pre": (dx * h2 / q2).sum(0)}
    dg = scale * n * e
    fold = lambda v: {"none": None, "channel": v.sum(0), "token": v.sum(1, keepdims=True), "full": v}[gate]  # noqa: E731
    out["d_gate"] = fold(dg)
    # What the roundings are relative to: the terms of each sum, which may cancel (in a row of one column they all do).
    terms = lambda g, v, q: (np.abs(g) + np.abs(v) / q * (np.abs(g * v) / q).sum(1, keepdims=True) / width) / q  # noqa: E731
    h2_terms = np.abs(f["h"]) + np.abs(h2 - f["h"])
    size = {"d_h": np.abs(dh) + terms(dx * one(f["w_pre"]), h2_terms, q2)}
    through_gate = np.abs(scale * one(f["gate"])) * size["d_h"]
    size |= {"d_y": terms(through_gate * np.abs(one(f["w_post"])), f["y"], q1), "d_w_post": (through_gate * np.abs(f["y"]) / q1).sum(0),
             "d_w_pre": np.abs(dx * h2_terms / q2).sum(0), "d_gate": fold(np.abs(scale * n) * size["d_h"])}
    return out, size


def numpy_of(t):
    return {k: None if v is None else v.double().numpy() for k, v in t.items()}


def on_gpu(t, apart=0):
    """The tensors on the GPU; matrices as rows of wider buffers where `apart`."""
    import torch
    out = {}
    for k, v in t.items():
        if v is not None and v.dim() == 2 and apart and v.shape[1] > 1:
            wide = torch.full((v.shape[0], v.shape[1] + 2 * apart), float("nan"), dtype=v.dtype, device="cuda")
            wide[:, apart:apart + v.shape[1]] = v.cuda()
            out[k] = wide[:, apart:apart + v.shape[1]]
        else:
            out[k] = None if v is None else v.cuda()
    return out


def near(got, want, name, what, slack=64.0, size=0.0):
    """Rounded once (UNIT), from fp32 values whose error is some roundings of the size of what was added up: a mean over
    the row, a root and a few products each side of it make a dozen, 64 are allowed for."""
    got = got.cpu().double().numpy()
    most = UNIT[name] * np.abs(want) * (1 + 1e-6) + slack * 2.0 ** -24 * (size + np.abs(want)) + TINY[name]
    worst = float(np.max(np.abs(got - want) / most)) if np.isfinite(got).all() else float("inf")
    assert worst <= 1, f"{what}: {worst:.3g} times what is allowed"


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("apart", [0, 3])
def test_forward_and_backward(name, gate, apart):
    for tokens, width in ((1, 1), (2, 7), (5, 64), (3, 511), (40, 513), (7, 2048), (600, 2050), (3, 4097), (2, 8192), (5, 8200), (2, 16384)):
        check_both_ways(tokens, width, name, gate, apart)


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("gate", GATES)
def test_rows_that_share_a_wavefront(name, gate):
    """narrow rows: several a workgroup, with some too few in the last one; at most 250 / 4 workgroups' sums of a column, in sixteen shares"""
    for tokens, width in ((1, 8), (9, 33), (1000, 64), (15, 65), (999, 100), (13, 128), (301, 129), (70, 200), (501, 256), (77, 257)):
        check_both_ways(tokens, width, name, gate, 0)
        check_both_ways(tokens, width, name, gate, 5)


def check_both_ways(tokens, width, name, gate, apart):
    import torch
    for weights in (True, False):
        print(f"[norms] {tokens} x {width} gate {gate} {name} weights {weights}", flush=True)
        t = inputs(tokens, width, name, gate, width + tokens, weights)
        d, f = on_gpu(t, apart), numpy_of(t)
        given = {k: d[k] for k in ("w_post", "w_pre", "gate")} | {"scale": 0.7}
        h_out, x_out = torch.empty_like(d["h"]), torch.empty_like(d["h"])
        rstd = torch.empty(tokens, 2, device="cuda")
        H.hbp_residual_norms(d["h"], d["y"], h_out, x_out, rstd=rstd, eps=EPS, **given)
        h2, x2, n, q1, q2 = forward(f, 0.7, EPS)
        near(h_out, h2, name, "h_out", size=np.abs(f["h"]) + np.abs(h2 - f["h"]))
        near(x_out, x2, name, "x_out", size=(np.abs(f["h"]) + np.abs(h2 - f["h"])) / q2 * (1.0 if f["w_pre"] is None else np.abs(f["w_pre"])))
        near(rstd, np.concatenate([1 / q1, 1 / q2], 1), "f32", "rstd")
        d_h, d_y, f32 = torch.empty_like(d["h"]), torch.empty_like(d["h"]), dict(dtype=torch.float32, device="cuda")
        d_gate = {"none": None, "channel": torch.full((width,), float("nan"), **f32), "token": torch.full((tokens, 1), float("nan"), **f32),
                  "full": torch.empty_like(d["gate"]) if gate == "full" else None}[gate]
        if gate == "token" and width == 1:
            d_gate = torch.empty_like(d["gate"])     # [tokens, 1] with one column: a full gate
        if gate == "full" and apart:
            d_gate = torch.empty_strided(d["gate"].shape, d["gate"].stride(), dtype=d["gate"].dtype, device="cuda")
        d_wp, d_wq = torch.full((width,), float("nan"), **f32), torch.full((width,), float("nan"), **f32)
        H.hbp_residual_norms_backward(d["d_h_out"], d["d_x_out"], d["h"], d["y"], rstd, d_h, d_y, d_w_post=d_wp, d_w_pre=d_wq, d_gate=d_gate, **given)
        want, size = backward(f, 0.7, EPS, gate)
        for key, got in (("d_h", d_h), ("d_y", d_y), ("d_w_post", d_wp), ("d_w_pre", d_wq), ("d_gate", d_gate)):
            if got is not None:
                near(got, want[key], {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}[got.dtype], key, size=size[key])


@pytest.mark.gpu
@pytest.mark.parametrize("gate", GATES)
def test_gradients_against_differences(gate):
    """d(sum of outputs times given weights) along random directions, by central differences of the 64-bit formula: error of order step^2."""
    import torch
    tokens, width, scale = 4, 37, -0.6
    t = inputs(tokens, width, "f32", gate, 5)
    f, d = numpy_of(t), on_gpu(t)
    given = {k: d[k] for k in ("w_post", "w_pre", "gate")} | {"scale": scale}
    rstd, ho, xo = torch.empty(tokens, 2, device="cuda"), torch.empty_like(d["h"]), torch.empty_like(d["h"])
    H.hbp_residual_norms(d["h"], d["y"], ho, xo, rstd=rstd, eps=EPS, **given)
    grads = {"h": torch.empty_like(d["h"]), "y": torch.empty_like(d["h"]), "w_post": torch.empty(width, device="cuda"), "w_pre": torch.empty(width, device="cuda"),
             "gate": None if gate == "none" else torch.empty_like(d["gate"])}
    H.hbp_residual_norms_backward(d["d_h_out"], d["d_x_out"], d["h"], d["y"], rstd, grads["h"], grads["y"], d_w_post=grads["w_post"],
                                  d_w_pre=grads["w_pre"], d_gate=grads["gate"], **given)

    def loss(v):
        h2, x2 = forward(v, scale, EPS)[:2]
        return (h2 * f["d_h_out"]).sum() + (x2 * f["d_x_out"]).sum()
    rng, step = np.random.default_rng(1), 1e-5
    for key, g in grads.items():
        if g is None:
            continue
        direction = rng.standard_normal(f[key].shape)
        difference = (loss(f | {key: f[key] + step * direction}) - loss(f | {key: f[key] - step * direction})) / (2 * step)
        along = (g.cpu().double().numpy() * direction).sum()
        assert abs(along - difference) <= 1e-5 * (np.abs(g.cpu().double().numpy() * direction).sum() + 1), key


@pytest.mark.gpu
def test_in_place_missing_gradients_and_no_tokens():
    import torch
    t = inputs(9, 300, "bf16", "token", 8)
    d = on_gpu(t)
    given = {k: d[k] for k in ("w_post", "w_pre", "gate")}
    ho, xo, rstd = torch.empty_like(d["h"]), torch.empty_like(d["h"]), torch.empty(9, 2, device="cuda")
    H.hbp_residual_norms(d["h"], d["y"], ho, xo, rstd=rstd, **given)
    h, y = d["h"].clone(), d["y"].clone()
    H.hbp_residual_norms(h, y, h, y, **given)      # h_out over h, x_out over y, no rstd
    assert torch.equal(h, ho) and torch.equal(y, xo)
    zero = torch.zeros_like(ho)
    for a, b in ((d["d_h_out"], None), (None, d["d_x_out"]), (None, None)):
        one, two = [torch.empty_like(ho), torch.empty_like(ho)], [torch.empty_like(ho), torch.empty_like(ho)]
        g1, g2 = torch.empty(9, 1, device="cuda"), torch.empty(9, 1, device="cuda")
        H.hbp_residual_norms_backward(a, b, d["h"], d["y"], rstd, *one, d_gate=g1, **given)
        H.hbp_residual_norms_backward(zero if a is None else a, zero if b is None else b, d["h"], d["y"], rstd, *two, d_gate=g2, **given)
        assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1]) and torch.equal(g1, g2)
    a, b = d["d_h_out"].clone(), d["d_x_out"].clone()
    want = [torch.empty_like(ho), torch.empty_like(ho)]
    H.hbp_residual_norms_backward(a, b, d["h"], d["y"], rstd, *want, **given)
    H.hbp_residual_norms_backward(a, b, d["h"], d["y"], rstd, a, b, **given)      # d_h over d_h_out, d_y over d_x_out
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])
    none = torch.empty(0, 300, dtype=torch.bfloat16, device="cuda")
    wp, wq, gg = (torch.full((300,), 5.0, device="cuda") for _ in range(3))
    H.hbp_residual_norms(none, none, none, none, gate=d["w_pre"])
    H.hbp_residual_norms_backward(none, none, none, none, torch.empty(0, 2, device="cuda"), none, none, d_w_post=wp, d_w_pre=wq, d_gate=gg, gate=d["w_pre"])
    assert not wp.any() and not wq.any() and not gg.any()


@pytest.mark.gpu
def test_rows_of_zeros_and_of_extremes():
    import torch
    h, y = torch.zeros(3, 100, device="cuda"), torch.zeros(3, 100, device="cuda")
    y[1] = 1e-30
    h[2], y[2] = 1e18, 1e18
    ho, xo, rstd = torch.empty_like(h), torch.empty_like(h), torch.empty(3, 2, device="cuda")
    H.hbp_residual_norms(h, y, ho, xo, rstd=rstd, eps=EPS)
    assert not ho[0].any() and not xo[0].any() and torch.isfinite(ho).all() and torch.isfinite(xo).all()
    assert np.allclose(xo[2].cpu().numpy(), 1.0, rtol=1e-6)
    dh, dy = torch.empty_like(h), torch.empty_like(h)
    H.hbp_residual_norms_backward(torch.ones_like(h), torch.ones_like(h), h, y, rstd, dh, dy)
    assert torch.isfinite(dh).all() and torch.isfinite(dy).all()
    assert np.allclose(dh[0].cpu().numpy(), 1 + EPS ** -0.5, rtol=1e-6)


@pytest.mark.gpu
def test_same_bits_on_a_stream_and_under_a_graph():
    import torch
    t = inputs(700, 1000, "f16", "channel", 20)
    d = on_gpu(t)
    given = {k: d[k] for k in ("w_post", "w_pre", "gate")}
    out = [torch.empty_like(d["h"]) for _ in range(4)] + [torch.empty(1000, device="cuda") for _ in range(3)]
    rstd = torch.empty(700, 2, device="cuda")

    def step(stream=None):
        H.hbp_residual_norms(d["h"], d["y"], out[0], out[1], rstd=rstd, stream=stream, **given)
        H.hbp_residual_norms_backward(d["d_h_out"], d["d_x_out"], d["h"], d["y"], rstd, out[2], out[3], d_w_post=out[4], d_w_pre=out[5], d_gate=out[6],
                                      stream=stream, **given)
    step()
    torch.cuda.synchronize()
    first = [o.clone() for o in out]
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        for o in out:
            o.zero_()
        side.wait_stream(torch.cuda.current_stream())
        step(stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, first))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        d["h"].copy_(t["h"] if k % 2 else -t["h"]), d["y"].copy_(t["y"] if k % 2 else -t["y"])
        step()
        torch.cuda.synchronize()
        eager = [o.clone() for o in out]
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))


@pytest.mark.gpu
def test_rows_further_apart_than_32_bits_count():
    import torch
    apart, width = (1 << 32) + 40, 96
    wide = torch.empty(apart + width, dtype=torch.float16, device="cuda")
    h = wide.as_strided((2, width), (apart, 1))
    t = inputs(2, width, "f16", "none", 30)
    h.copy_(t["h"])
    d = on_gpu(t)
    ho, xo, rstd, want = torch.empty_like(d["y"]), torch.empty_like(d["y"]), torch.empty(2, 2, device="cuda"), torch.empty_like(d["y"])
    H.hbp_residual_norms(d["h"], d["y"], want, xo)
    H.hbp_residual_norms(h, d["y"], ho, xo, rstd=rstd)
    assert torch.equal(ho, want)
    dh, dy, dh2, dy2 = (torch.empty_like(d["y"]) for _ in range(4))
    H.hbp_residual_norms_backward(d["d_h_out"], d["d_x_out"], h, d["y"], rstd, dh, dy)
    H.hbp_residual_norms_backward(d["d_h_out"], d["d_x_out"], d["h"], d["y"], rstd, dh2, dy2)
    assert torch.equal(dh, dh2) and torch.equal(dy, dy2)


@pytest.mark.gpu
def test_what_the_binding_refuses():
    import torch
    h, y = torch.zeros(4, 32, device="cuda"), torch.zeros(4, 32, device="cuda")
    good = dict(h=h, y=y, h_out=torch.zeros_like(h), x_out=torch.zeros_like(h))
    for change in (dict(y=y.half()), dict(y=y[:3]), dict(h=h.double()), dict(h=h.cpu()), dict(h_out=h.t()), dict(gate=torch.zeros(31, device="cuda")),
                   dict(gate=torch.zeros(3, 1, device="cuda")), dict(gate=torch.zeros(4, 32, device="cuda", dtype=torch.float16)),
                   dict(w_post=torch.zeros(33, device="cuda")), dict(rstd=torch.zeros(4, device="cuda")), dict(x_out=h[:1].expand(4, 32))):
        with pytest.raises(AssertionError):
            H.hbp_residual_norms(**good | change)
    for change, status in ((dict(eps=0.0), -1), (dict(eps=float("nan")), -1)):
        with pytest.raises(H.HbpError) as e:
            H.hbp_residual_norms(**good | change)
        assert e.value.status == status
    big = torch.zeros(1, 16385, device="cuda")
    with pytest.raises(H.HbpError) as e:
        H.hbp_residual_norms(big, big, torch.empty_like(big), torch.empty_like(big))
    assert e.value.status == -4
    with pytest.raises(AssertionError):   # no gate, but a gradient for one
        H.hbp_residual_norms_backward(h, h, h, y, torch.zeros(4, 2, device="cuda"), h, y, d_gate=torch.zeros(32, device="cuda"))


def test_what_the_library_refuses():
    L = H.lib()
    at = 4096

    def n(tokens=2, width=8, kind=0, gate_kind=0, w_post=None, w_pre=None, gate=None, ldg=0, eps=1e-6):
        return H.hbp_norms_t(tokens, width, kind, gate_kind, w_post, w_pre, gate, ldg, 1.0, eps)
    call = lambda n_, h=at, ldh=8, y=at, ldy=8, ho=at, ldho=8, xo=at, ldxo=8, rstd=None: L.hbp_residual_norms(n_, h, ldh, y, ldy, ho, ldho, xo, ldxo, rstd, None)  # noqa: E731
    for bad in (n(tokens=-1), n(width=0), n(kind=3), n(kind=-1), n(gate_kind=4, gate=at), n(gate_kind=1), n(gate=at), n(gate_kind=3, gate=at, ldg=7), n(eps=0.0),
                n(eps=-1.0), n(w_post=4098), n(w_pre=4097), n(gate=4097, gate_kind=2)):
        assert call(bad) == -1
    assert call(None) == -1 and call(n(width=16385)) == -4 and call(n(tokens=0)) == 0
    for change in (dict(h=None), dict(y=None), dict(ho=None), dict(xo=None), dict(ldh=7), dict(ldy=7), dict(ldho=7), dict(ldxo=7), dict(h=4098), dict(rstd=4097)):
        assert call(n(), **change) == -1
    need = ctypes.c_size_t()
    assert L.hbp_residual_norms_backward_workspace(n(), need) == 0 and need.value > 0
    assert L.hbp_residual_norms_backward_workspace(n(), None) == -1
    back = lambda n_, size, ws=4096, **k: L.hbp_residual_norms_backward(n_, k.get("dho", at), 8, at, 8, k.get("h", at), 8, at, 8, k.get("rstd", at),  # noqa: E731
                                                                       k.get("dh", at), 8, at, k.get("lddy", 8), None, None, k.get("dg"), ws, size, None)
    assert back(n(), need.value - 1) == -1 and back(n(), need.value, ws=None) == -1 and back(n(), need.value, ws=4100) == -1
    for change in (dict(h=None), dict(rstd=None), dict(dh=None), dict(lddy=7), dict(dg=at), dict(dho=4098)):
        assert back(n(), need.value, **change) == -1


@pytest.mark.gpu
def test_narrow_rows_in_place():
    import torch
    for tokens, width in ((9, 40), (3, 128), (5, 250)):
        d = on_gpu(inputs(tokens, width, "f16", "full", 8))
        given = {k: d[k] for k in ("w_post", "w_pre", "gate")}
        ho, xo, rstd = torch.empty_like(d["h"]), torch.empty_like(d["h"]), torch.empty(tokens, 2, device="cuda")
        H.hbp_residual_norms(d["h"], d["y"], ho, xo, rstd=rstd, **given)
        h, y = d["h"].clone(), d["y"].clone()
        H.hbp_residual_norms(h, y, h, y, **given)
        assert torch.equal(h, ho) and torch.equal(y, xo)
        want, a, b = [torch.empty_like(ho), torch.empty_like(ho)], d["d_h_out"].clone(), d["d_x_out"].clone()
        H.hbp_residual_norms_backward(a, b, d["h"], d["y"], rstd, *want, **given)
        H.hbp_residual_norms_backward(a, b, d["h"], d["y"], rstd, a, b, **given)
        assert torch.equal(a, want[0]) and torch.equal(b, want[1])


@pytest.mark.gpu
def test_gates_of_other_dimensions_are_refused():
    import torch
    h = torch.zeros(4, 32, device="cuda")
    for gate in (torch.zeros((), device="cuda"), torch.zeros(4, 1, 1, device="cuda"), torch.zeros(1, 4, 32, device="cuda")):
        with pytest.raises(AssertionError):
            H.hbp_residual_norms(h, h, torch.empty_like(h), torch.empty_like(h), gate=gate)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("gate", GATES)
def test_gradients_of_large_rows_and_of_rows_of_zeros_with_a_small_eps(name, gate):
    """Norms' factors from 1e-17 to 1e17 (their cubes are no fp32 numbers), with nothing but the norms' own terms in the gradients, too: the bounds are those of
    ordinary rows, whose roundings are relative to the terms that are added."""
    import torch
    for width in (40, 300, 2050):
        for size_h, size_y, eps in ((1e14, 1e14, EPS), (1e17, 1.0, EPS), (1.0, 1e17, EPS), (1e17, 1e17, EPS), (0.0, 0.0, 1e-28), (0.0, 0.0, 1e-34), (1.0, 0.0, 1e-28)):
            print(f"[norms] {width} gate {gate} {name} h {size_h} y {size_y} eps {eps}", flush=True)
            t = inputs(6, width, name, gate, width)
            t["h"], t["y"] = t["h"] * size_h, t["y"] * size_y
            t["h"][5], t["y"][5] = some_x(1, width, name, 77)[0], some_x(1, width, name, 78)[0]    # an ordinary row in the same batch
            for alone in (False, True):
                if alone:
                    t["d_h_out"] = torch.zeros_like(t["d_h_out"])
                d, f = on_gpu(t), numpy_of(t)
                given = {k: d[k] for k in ("w_post", "w_pre", "gate")} | {"scale": 0.7}
                rstd, out = torch.empty(6, 2, device="cuda"), [torch.empty_like(d["h"]) for _ in range(4)]
                H.hbp_residual_norms(d["h"], d["y"], out[0], out[1], rstd=rstd, eps=eps, **given)
                d_wp, d_wq = torch.empty(width, device="cuda"), torch.empty(width, device="cuda")
                d_gate = {"none": None, "channel": torch.empty(width, device="cuda"), "token": torch.empty(6, 1, device="cuda"), "full": torch.empty_like(d["h"])}[gate]
                H.hbp_residual_norms_backward(d["d_h_out"], d["d_x_out"], d["h"], d["y"], rstd, out[2], out[3], d_w_post=d_wp, d_w_pre=d_wq, d_gate=d_gate, **given)
                want, size = backward(f, 0.7, eps, gate)
                for key, got in (("d_h", out[2]), ("d_y", out[3]), ("d_w_post", d_wp), ("d_w_pre", d_wq), ("d_gate", d_gate)):
                    if got is not None:
                        near(got, want[key], "bf16" if got.dtype == torch.bfloat16 else "f32", key, size=size[key])


@pytest.mark.gpu
@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("tokens,width", [((1 << 24) + 13, 1), ((1 << 21) + 3, 300)])
def test_more_rows_than_one_launch_takes(tokens, width, gate):
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    h, y = r(tokens, width), r(tokens, width)
    gates = {"none": None, "channel": r(width), "token": r(tokens, 1), "full": r(tokens, width)}[gate]
    ho, xo, rstd = torch.empty_like(h), torch.empty_like(h), torch.empty(tokens, 2, device="cuda")
    print(f"[norms] {tokens} x {width} {gate}", flush=True)
    H.hbp_residual_norms(h, y, ho, xo, rstd=rstd, gate=gates, eps=EPS)
    for part in (slice(0, 50), slice(tokens - 100, tokens)):
        cut = None if gates is None else gates if gate == "channel" else gates[part]
        a, b, factors = torch.empty_like(h[part]), torch.empty_like(h[part]), torch.empty_like(rstd[part])
        H.hbp_residual_norms(h[part], y[part], a, b, rstd=factors, gate=cut, eps=EPS)
        assert torch.equal(ho[part], a) and torch.equal(xo[part], b) and torch.equal(rstd[part], factors)


@pytest.mark.gpu
def test_more_threads_than_32_bits_count():
    import torch
    tokens = (1 << 29) + 5
    h, y = torch.ones(tokens, 1, dtype=torch.bfloat16, device="cuda"), torch.ones(tokens, 1, dtype=torch.bfloat16, device="cuda")
    print("[norms] 2^29 + 5 rows of one column", flush=True)
    H.hbp_residual_norms(h, y, h, y, eps=EPS)
    assert (h == 2).all() and (y == 1).all()
