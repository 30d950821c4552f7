"""Matrices held in 4 bits: packing, products with one and with many vectors, transposed products, against numpy in 64 bits."""
import ctypes

import numpy as np
import pytest

import paper_2504_08860_amd as H

TYPES = ["f32", "f16", "bf16"]
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}  # half a step between neighbours, relative
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}


def dtype(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def matrix(rows, cols, group, scales, zeros, seed, spread=0.5):
    """(codes, scales, zero points or None on the GPU, the values in 64 bits)"""
    import torch
    rng = np.random.default_rng(seed)
    codes_shape, scales_shape = H.hbp_q4_shapes(rows, cols, group)
    codes = torch.from_numpy(rng.integers(0, 256, codes_shape, dtype=np.uint8))   # (what lies behind the last column is anything)
    s = torch.from_numpy((0.02 * (1 + spread * rng.uniform(-1, 1, scales_shape))).astype(np.float32)).to(dtype(scales))
    z = torch.from_numpy(rng.integers(4, 12, scales_shape).astype(np.float32)).to(dtype(scales)) if zeros else None
    return codes.cuda(), s.cuda(), None if z is None else z.cuda(), values(codes, s, z, cols, group)


def values(codes, s, z, cols, group):
    c = codes.cpu().numpy()
    q = np.stack([c & 15, c >> 4], axis=2).reshape(c.shape[0], -1)[:, :cols].astype(np.float64)
    of = np.arange(cols) // group
    s = s.cpu().double().numpy()[:, of]
    return s * (q - (8.0 if z is None else z.cpu().double().numpy()[:, of]))


def some_x(vectors, n, name, seed):
    import torch
    return torch.from_numpy(np.random.default_rng(seed).standard_normal((vectors, n)).astype(np.float32)).to(dtype(name))


def agree(y, want, x, name, top_scale=0.03, what=""):
    """Every output is rounded once (UNIT) and is a sum of products s (c - z) x that fp32 holds to 2^-24 of partial sums of up to
    32 s times those of x, whose size is that of |x|_2 where x has either sign: sixteen such roundings are allowed for."""
    got = y.cpu().double().numpy()
    size = np.sqrt((x.cpu().double().numpy() ** 2).sum(axis=1, keepdims=True))
    most = UNIT[name] * np.abs(want) + 16 * 32 * 2.0 ** -24 * top_scale * size + TINY[name]
    worst = float(np.max(np.abs(got - want) / most)) if np.isfinite(got).all() else float("inf")
    assert worst <= 1, f"{what}: {worst:.3g} times what is allowed"


# one column, a part of a group, odd and whole sizes; one row, part of a tile of rows, several workgroups
SHAPES = [(1, 1), (1, 31), (3, 33), (16, 32), (17, 100), (64, 128), (100, 257), (129, 1000), (300, 2080), (257, 4099), (1000, 512)]


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("vectors", [1, 2, 3, 5, 8, 9, 16, 17, 33, 64, 70])
@pytest.mark.parametrize("direction", ["mv", "mv_t"])
def test_products(name, vectors, direction):
    import torch
    for k, (rows, cols) in enumerate(SHAPES):
        group = [32, 64, 128, 256, 512][(k + vectors) % 5]
        scales, zeros = TYPES[(k + vectors) % 3], (k + vectors) % 2 == 0
        print(f"[q4 {direction}] {rows} x {cols} group {group} {scales} zeros {zeros} {vectors} of {name}", flush=True)
        c, s, z, w = matrix(rows, cols, group, scales, zeros, 7 * k + vectors)
        n_in, n_out = (cols, rows) if direction == "mv" else (rows, cols)
        x = some_x(vectors, n_in, name, k)
        y = torch.full((vectors, n_out), float("nan"), dtype=dtype(name), device="cuda")
        call = H.hbp_q4_mv if direction == "mv" else H.hbp_q4_mv_t
        call(c, s, x.cuda(), y, group=group, zeros=z)
        xd = x.double().numpy()
        agree(y, xd @ w.T if direction == "mv" else xd @ w, x, name, what=f"{rows}x{cols}")


@pytest.mark.gpu
@pytest.mark.parametrize("scales", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128, 256, 512])
@pytest.mark.parametrize("zeros", [False, True])
def test_every_group_and_scale_type(scales, group, zeros):
    import torch
    rows, cols = 210, 1111
    c, s, z, w = matrix(rows, cols, group, scales, zeros, group)
    for vectors in (1, 4, 6, 40):
        for name in TYPES:
            print(f"[q4 groups] {group} {scales} zeros {zeros} {vectors} of {name}", flush=True)
            x, g = some_x(vectors, cols, name, 1), some_x(vectors, rows, name, 2)
            y, d = torch.empty(vectors, rows, dtype=x.dtype, device="cuda"), torch.empty(vectors, cols, dtype=x.dtype, device="cuda")
            H.hbp_q4_mv(c, s, x.cuda(), y, group=group, zeros=z)
            H.hbp_q4_mv_t(c, s, g.cuda(), d, group=group, zeros=z)
            agree(y, x.double().numpy() @ w.T, x, name, what="mv")
            agree(d, g.double().numpy() @ w, g, name, what="mv_t")


@pytest.mark.gpu
@pytest.mark.parametrize("direction", ["mv", "mv_t"])
def test_strides_one_dimension_and_a_stream(direction):
    """Rows of wider buffers at odd places, vectors as such, another stream, and the outputs' surroundings left alone."""
    import torch
    rows, cols, group = 130, 515, 32
    c, s, z, w = matrix(rows, cols, group, "f16", True, 3)
    call = H.hbp_q4_mv if direction == "mv" else H.hbp_q4_mv_t
    n_in, n_out = (cols, rows) if direction == "mv" else (rows, cols)
    m = w.T if direction == "mv" else w
    for name in TYPES:
        for vectors in (1, 3, 20):
            wide_x = torch.full((vectors, n_in + 7), float("nan"), dtype=dtype(name), device="cuda")
            wide_y = torch.full((vectors, n_out + 9), 77.0, dtype=dtype(name), device="cuda")
            x, y = wide_x[:, 3:3 + n_in], wide_y[:, 5:5 + n_out]
            x.copy_(some_x(vectors, n_in, name, 4))
            print(f"[q4 strides] {direction} {vectors} of {name}", flush=True)
            call(c, s, x, y, group=group, zeros=z)
            agree(y, x.cpu().double().numpy() @ m, x, name)
            assert (wide_y[:, :5] == 77).all() and (wide_y[:, 5 + n_out:] == 77).all()
            one = torch.empty(n_out, dtype=x.dtype, device="cuda")
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            for stream in (side, side.cuda_stream):
                one.zero_()
                side.wait_stream(torch.cuda.current_stream())
                call(c, s, x[0], one, group=group, zeros=z, stream=stream)
                torch.cuda.synchronize()
                agree(one[None], x[:1].cpu().double().numpy() @ m, x[:1], name)


@pytest.mark.gpu
@pytest.mark.parametrize("direction", ["mv", "mv_t"])
@pytest.mark.parametrize("name", TYPES)
def test_infinities_and_large_values_are_what_the_sum_makes_of_them(direction, name):
    """An infinite x times a weight that is not 0 is an infinity of its sign, times a weight of 0 a NaN; finite values whose sum is
    finite give it, however large they are."""
    import torch
    rows, cols, group = 70, 300, 64
    c, s, z, w = matrix(rows, cols, group, "f32", False, 5, spread=0.0)
    n_in, n_out = (cols, rows) if direction == "mv" else (rows, cols)
    m = w.T if direction == "mv" else w
    call = H.hbp_q4_mv if direction == "mv" else H.hbp_q4_mv_t
    x = some_x(4, n_in, name, 6)
    x[0, 33] = float("inf")
    x[1, 1] = float("nan")
    x[2] = 0
    x[2, 7] = torch.finfo(x.dtype).max / 4
    y = torch.empty(4, n_out, dtype=x.dtype, device="cuda")
    for vectors in (4, 1):
        call(c, s, x[:vectors].cuda(), y[:vectors], group=group, zeros=z)
        got = y[:vectors].cpu().double().numpy()
        sign = np.where(m[33] > 0, np.inf, np.where(m[33] < 0, -np.inf, np.nan))
        assert np.array_equal(got[0], sign, equal_nan=True)
    call(c, s, x.cuda(), y, group=group, zeros=z)
    got = y.cpu().double().numpy()
    assert np.isnan(got[1]).all()
    want = x[2].double().numpy() @ m
    assert np.isfinite(got[2]).all() and (np.abs(got[2] - want) <= 2 * UNIT[name] * np.abs(want) + 2.0 ** -20 * np.abs(want).max()).all()
    agree(y[3:], x[3:].double().numpy() @ m, x[3:], name)


@pytest.mark.gpu
def test_more_codes_than_32_bits_count():
    import torch
    rows, cols = 69_999, 131_072
    codes = torch.randint(0, 256, H.hbp_q4_shapes(rows, cols, 512)[0], dtype=torch.uint8, device="cuda")
    assert codes.numel() > 1 << 32
    s = torch.full(H.hbp_q4_shapes(rows, cols, 512)[1], 0.02, device="cuda")
    x = some_x(1, cols, "bf16", 8)
    y = torch.empty(1, rows, dtype=x.dtype, device="cuda")
    print("[q4 large] mv", flush=True)
    H.hbp_q4_mv(codes, s, x.cuda(), y, group=512)
    for part in (slice(0, 40), slice(rows - 40, rows)):
        agree(y[:, part], x.double().numpy() @ values(codes[part], s[part], None, cols, 512).T, x, "bf16")
    g = torch.zeros(1, rows, dtype=x.dtype)
    g[0, -40:] = some_x(1, 40, "bf16", 9)[0]
    d = torch.empty(1, cols, dtype=x.dtype, device="cuda")
    print("[q4 large] mv_t", flush=True)
    H.hbp_q4_mv_t(codes, s, g.cuda(), d, group=512)
    agree(d, g[:, -40:].double().numpy() @ values(codes[-40:], s[-40:], None, cols, 512), g, "bf16")


@pytest.mark.gpu
def test_the_transposed_product_is_the_gradient():
    """By differences of the product in its fp32 form: it is linear, so a difference over one coordinate is the weight itself."""
    import torch
    rows, cols, group = 40, 96, 32
    c, s, z, w = matrix(rows, cols, group, "f32", True, 11)
    g = some_x(1, rows, "f32", 12).cuda()
    x = torch.zeros(cols + 1, cols, device="cuda")
    x[1:] = torch.eye(cols, device="cuda")
    y = torch.empty(cols + 1, rows, device="cuda")
    d = torch.empty(1, cols, device="cuda")
    H.hbp_q4_mv(c, s, x, y, group=group, zeros=z)
    H.hbp_q4_mv_t(c, s, g, d, group=group, zeros=z)
    difference = ((y[1:] - y[:1]).cpu().double() @ g[0].cpu().double()).numpy()
    assert np.abs(d[0].cpu().double().numpy() - difference).max() <= 2.0 ** -24 * 64 * np.abs(w).max() * np.abs(g.cpu().numpy()).sum()


@pytest.mark.gpu
def test_same_bits_every_time_and_under_a_graph():
    import torch
    rows, cols, group = 700, 1500, 128
    c, s, z, w = matrix(rows, cols, group, "bf16", False, 13)
    for vectors in (1, 24):
        x, g = some_x(vectors, cols, "f32", 14).cuda(), some_x(vectors, rows, "f32", 15).cuda()
        y, d = torch.empty(vectors, rows, device="cuda"), torch.empty(vectors, cols, device="cuda")

        def both():
            H.hbp_q4_mv(c, s, x, y, group=group, zeros=z)
            H.hbp_q4_mv_t(c, s, g, d, group=group, zeros=z)
        both()
        torch.cuda.synchronize()
        first = y.clone(), d.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both()
        for _ in range(3):
            y.zero_(), d.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, first[0]) and torch.equal(d, first[1])
            x.mul_(2), g.mul_(2)     # (a power of two: the same bits one exponent up)
            both()
            torch.cuda.synchronize()
            assert torch.equal(y, 2 * first[0]) and torch.equal(d, 2 * first[1])
            first = y.clone(), d.clone()


def pack_in_numpy(w, group, scales, zeros):
    """The rule of the header in fp32, group by group."""
    import torch
    rows, cols = w.shape
    groups = (cols + group - 1) // group
    codes, s_all, z_all = np.zeros((rows, cols), np.int64), np.zeros((rows, groups), np.float32), np.zeros((rows, groups), np.float32)
    rounded = lambda v: torch.from_numpy(v.astype(np.float32)).to(dtype(scales)).float().numpy()  # noqa: E731
    for k in range(groups):
        part = w[:, k * group:(k + 1) * group].astype(np.float32)
        low, high = np.minimum(part.min(1), 0), np.maximum(part.max(1), 0)
        wide = (high - low) * np.float32(1 / 15) if zeros else np.maximum(-low, high) * np.float32(1 / 7)
        s = rounded(np.minimum(wide, np.float32(torch.finfo(dtype(scales)).max)))
        with np.errstate(divide="ignore", invalid="ignore"):
            z = np.where(s == 0, np.float32(0), np.rint(-low / s)) if zeros else np.full_like(s, 8)
            q = np.where(s[:, None] == 0, z[:, None], np.rint(part / s[:, None] + z[:, None]))
        codes[:, k * group:(k + 1) * group] = np.clip(q, 0, 15)
        s_all[:, k], z_all[:, k] = s, z
    return codes, s_all, z_all


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("scales", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
def test_pack_and_unpack(name, scales, zeros):
    import torch
    for rows, cols, group in ((1, 1, 32), (5, 33, 32), (3, 64, 64), (17, 200, 128), (33, 2047, 256), (9, 4100, 512)):
        print(f"[q4 pack] {rows} x {cols} group {group} {name} {scales} zeros {zeros}", flush=True)
        wide = some_x(rows, cols + 3, name, cols).cuda()
        w = wide[:, 1:1 + cols]
        w[0] = 0                                  # groups of nothing but zeros
        if rows > 2:
            w[1] = 3.0                            # of one value
            w[2] = w[2].abs()                     # of one sign
        codes_shape, scales_shape = H.hbp_q4_shapes(rows, cols, group)
        c = torch.full(codes_shape, 255, dtype=torch.uint8, device="cuda")
        s = torch.full(scales_shape, float("nan"), dtype=dtype(scales), device="cuda")
        z = torch.full_like(s, float("nan")) if zeros else None
        H.hbp_q4_pack(w, c, s, group=group, zeros=z)
        codes, s_want, z_want = pack_in_numpy(w.float().cpu().numpy(), group, scales, zeros)
        got = c.cpu().numpy()
        both = np.stack([got & 15, got >> 4], axis=2).reshape(rows, -1)
        assert np.array_equal(both[:, :cols], codes) and not both[:, cols:].any()
        assert np.array_equal(s.float().cpu().numpy(), s_want)
        if zeros:
            assert np.array_equal(z.float().cpu().numpy(), z_want)
        for out_name in TYPES:
            out = torch.full((rows, cols + 5), 7.0, dtype=dtype(out_name), device="cuda")
            H.hbp_q4_unpack(c, s, cols, group=group, zeros=z, out=out[:, 2:2 + cols])
            of = np.arange(cols) // group
            back = torch.from_numpy((codes - z_want[:, of]).astype(np.float32) * s_want[:, of]).to(dtype(out_name))
            assert torch.equal(out[:, 2:2 + cols].cpu(), back) and (out[:, :2] == 7).all() and (out[:, 2 + cols:] == 7).all()
        assert torch.equal(H.hbp_q4_unpack(c, s, cols, group=group, zeros=z).cpu(),
                           torch.from_numpy((codes - z_want[:, of]).astype(np.float32) * s_want[:, of]))


@pytest.mark.gpu
@pytest.mark.parametrize("zeros", [False, True])
def test_pack_of_values_that_no_scale_fits(zeros):
    import torch
    w = some_x(4, 128, "f32", 3).cuda()
    w[0, 40], w[1, 100], w[2, 3] = float("nan"), float("inf"), 3e38
    codes_shape, scales_shape = H.hbp_q4_shapes(4, 128, 32)
    for scales in TYPES:
        c, s = torch.empty(codes_shape, dtype=torch.uint8, device="cuda"), torch.empty(scales_shape, dtype=dtype(scales), device="cuda")
        z = torch.empty_like(s) if zeros else None
        H.hbp_q4_pack(w, c, s, group=32, zeros=z)
        nan = torch.isnan(s).cpu().numpy()
        want = np.zeros((4, 4), bool)
        want[0, 1] = want[1, 3] = True
        assert np.array_equal(nan, want) and torch.isfinite(s[~torch.isnan(s)]).all()
        out = H.hbp_q4_unpack(c, s, 128, group=32, zeros=z)
        assert torch.isnan(out[0, 32:64]).all() and torch.isnan(out[1, 96:]).all() and torch.isfinite(out[2:]).all()


@pytest.mark.gpu
def test_no_vectors_at_all():
    import torch
    c, s, z, _ = matrix(20, 40, 32, "f32", False, 1)
    for name in TYPES:
        x, y = torch.empty(0, 40, dtype=dtype(name), device="cuda"), torch.empty(0, 20, dtype=dtype(name), device="cuda")
        H.hbp_q4_mv(c, s, x, y, group=32)
        H.hbp_q4_mv_t(c, s, y, x, group=32)
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_what_the_binding_refuses():
    import torch
    c, s, z, _ = matrix(20, 40, 32, "f32", False, 1)
    x, y = torch.zeros(2, 40, device="cuda"), torch.zeros(2, 20, device="cuda")
    wrong = [dict(codes=c[:, :-1]), dict(codes=c.int()), dict(scales=s[:, :1]), dict(scales=s.double()), dict(x=x.double()), dict(x=x.half()),
             dict(x=x.cpu()), dict(x=x[:1]), dict(y=y[:, :-1]), dict(y=y.cpu()), dict(x=x.t().contiguous().t()), dict(x=x[:1].expand(2, 40)),
             dict(group=64), dict(group=0), dict(zeros=s.half()), dict(zeros=s[:-1]), dict(x=x[0])]
    for change in wrong:
        a = dict(codes=c, scales=s, x=x, y=y, group=32, zeros=None) | change
        with pytest.raises(AssertionError):
            H.hbp_q4_mv(**a)
    with pytest.raises(H.HbpError) as e:   # a group that the library does not know
        H.hbp_q4_mv(c, torch.zeros(20, 3, device="cuda"), x, y, group=16)
    assert e.value.status == -1
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    with pytest.raises(H.HbpError):
        H.hbp_q4_mv_t(c, s, y, x, group=32, workspace=small)


def test_what_the_library_refuses():
    """Before anything is launched: this runs without a GPU."""
    L = H.lib()
    at = lambda n: ctypes.c_void_p(n)  # noqa: E731

    def m(codes=4096, scales=4096, zeros=None, rows=8, cols=64, group=32, kind=0):
        return H.hbp_q4_matrix_t(codes, scales, zeros, rows, cols, group, kind)
    good = dict(type=0, x=at(4096), ldx=64, y=at(8192), ldy=8, vectors=2)
    bad = [(m(codes=None), {}), (m(scales=None), {}), (m(codes=4104), {}), (m(scales=4098), {}), (m(zeros=4097, kind=1), {}), (m(rows=0), {}), (m(cols=0), {}),
           (m(group=16), {}), (m(group=33), {}), (m(group=1024), {}), (m(kind=3), {}), (m(), dict(type=5)), (m(), dict(x=None)), (m(), dict(y=None)),
           (m(), dict(ldx=63)), (m(), dict(ldy=7)), (m(), dict(vectors=-1)), (m(), dict(x=at(4098))), (m(), dict(y=at(8193)))]
    for matrix_, change in bad:
        a = good | change
        assert L.hbp_q4_mv(matrix_, a["type"], a["x"], a["ldx"], a["y"], a["ldy"], a["vectors"], None) == -1, change
    assert L.hbp_q4_mv(m(rows=1 << 31), 0, at(4096), 64, at(4096), 1 << 31, 1, None) == -4
    assert L.hbp_q4_mv(m(cols=(1 << 28) + 1), 0, at(4096), 1 << 29, at(4096), 8, 1, None) == -4
    assert L.hbp_q4_mv(m(), 0, at(4096), 64, at(8192), 8, (1 << 24) + 1, None) == -4
    assert L.hbp_q4_mv(None, 0, at(4096), 64, at(4096), 8, 1, None) == -1
    assert L.hbp_q4_mv(m(), 0, None, 64, None, 8, 0, None) == 0
    need = ctypes.c_size_t()
    assert L.hbp_q4_mv_t_workspace(m(), 3, need) == 0 and L.hbp_q4_mv_t_workspace(m(), -1, need) == -1 and L.hbp_q4_mv_t_workspace(m(), 3, None) == -1
    assert L.hbp_q4_mv_t_workspace(m(), (1 << 24) + 1, need) == -4
    for matrix_, change in bad:
        if not change:
            assert L.hbp_q4_pack(matrix_, 0, at(4096), 64, None) == -1
            assert L.hbp_q4_unpack(matrix_, 0, at(4096), 64, None) == -1
    assert L.hbp_q4_pack(m(), 0, None, 64, None) == -1 and L.hbp_q4_pack(m(), 0, at(4096), 63, None) == -1


@pytest.mark.gpu
def test_tensors_of_other_dimensions_are_refused():
    import torch
    c, s, _, _ = matrix(20, 40, 32, "f32", False, 1)
    x, y, one = torch.zeros(40, device="cuda"), torch.zeros(20, device="cuda"), torch.zeros((), device="cuda")
    for change in (dict(codes=c[0, 0]), dict(codes=c.flatten()), dict(scales=s.flatten()), dict(x=one), dict(y=one), dict(x=x.view(1, 1, 40))):
        a = dict(codes=c, scales=s, x=x, y=y, group=32) | change
        with pytest.raises(AssertionError):
            H.hbp_q4_mv(**a)
        with pytest.raises(AssertionError):
            H.hbp_q4_mv_t(**a | dict(x=a["y"], y=a["x"]))


def codes_around_their_zeros(rows, cols, group, scales, zeros, seed):
    """(codes, scales, zero points or None, values in 64 bits), on the GPU: of every weight its opposite is as likely, so that a sum of them with numbers of one sign
    is as large as a sum with numbers of either."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape, of = H.hbp_q4_shapes(rows, cols, group)[1], torch.arange(cols, device="cuda") // group
    z = torch.randint(4, 12, shape, generator=g, device="cuda") if zeros else torch.full(shape, 8, device="cuda")
    q = z[:, of] + torch.randint(-4, 5, (rows, cols), generator=g, device="cuda")
    packed = torch.zeros(rows, (cols + 31) // 32 * 32, dtype=torch.uint8, device="cuda")
    packed[:, :cols] = q.to(torch.uint8)
    s = (0.02 * (0.5 + torch.rand(shape, generator=g, device="cuda"))).to(dtype(scales))
    z = z.to(dtype(scales))
    if zeros == "broken":                     # zero points between codes
        z = (z.float() + 0.3).to(dtype(scales))
    w = s.double()[:, of] * (q.double() - z.double()[:, of])
    return packed[:, 0::2] | packed[:, 1::2] << 4, s, z if zeros else None, w


X_OF_ONE_SIGN = {"positive": lambda n: n.abs(), "cut off": lambda n: n.clamp(min=0), "around 3": lambda n: n.abs() + 3}


def near_the_sum(y, x, w, roundings, what):
    """fp32 sums of products w x (x [vectors, n], w [n, outputs], 64 bits, on the GPU): so many roundings of the size of the sum and of the root of its terms' squares,
    which is the size of partial sums of terms of either sign."""
    import torch
    want, terms = torch.mm(x, w), torch.mm(x.square(), w.square()).sqrt()
    worst = ((y.double() - want).abs() / (2.0 ** -24 * (want.abs() + terms))).max().item()
    assert worst <= roundings, f"{what}: {worst:.3g} roundings, {roundings:.3g} allowed"


@pytest.mark.gpu
@pytest.mark.parametrize("kind", list(X_OF_ONE_SIGN))
@pytest.mark.parametrize("zeros", [False, True, "broken"])
def test_products_with_an_x_that_is_not_centred(kind, zeros):
    """Sums over a group, then over groups, of terms that are centred though x is not: sixteen roundings, whichever kernel it is (in a model of the sums, fp32 in pieces of
    eight columns, it is up to eight)."""
    import torch
    for rows, cols in ((300, 4096), (8300, 2048)):
        for group in (32, 64, 128, 512):
            c, s, z, w = codes_around_their_zeros(rows, cols, group, "f32" if group == 64 else "f16", zeros, group)
            wt = w.t().contiguous()
            for vectors in (1, 5, 9, 21):
                print(f"[q4 not centred] mv {rows} x {cols} group {group} zeros {zeros} {kind} {vectors}", flush=True)
                x = X_OF_ONE_SIGN[kind](torch.randn(vectors, cols, generator=torch.Generator(device="cuda").manual_seed(vectors), device="cuda"))
                y = torch.empty(vectors, rows, device="cuda")
                H.hbp_q4_mv(c, s, x, y, group=group, zeros=z)
                near_the_sum(y, x.double(), wt, 16, f"{rows} x {cols} group {group} {vectors} vectors")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", list(X_OF_ONE_SIGN))
@pytest.mark.parametrize("zeros", [False, True, "broken"])
def test_transposed_products_with_an_x_that_is_not_centred(kind, zeros):
    """One row after another in fp32: roundings by the root of the number of rows, half of it and sixteen more are allowed (in a model of the sums it is up to a
    fifth of the root)."""
    import torch
    for rows, cols, group, vectors in ((8192, 300, 128, 1), (8192, 515, 32, 19), (8192, 2048, 64, 640), (1500, 300, 128, 4), (6001, 1000, 512, 2)):
        print(f"[q4 not centred] mv_t {rows} x {cols} group {group} zeros {zeros} {kind} {vectors}", flush=True)
        c, s, z, w = codes_around_their_zeros(rows, cols, group, "f32" if group == 64 else "f16", zeros, group)
        x = X_OF_ONE_SIGN[kind](torch.randn(vectors, rows, generator=torch.Generator(device="cuda").manual_seed(vectors), device="cuda"))
        y = torch.empty(vectors, cols, device="cuda")
        H.hbp_q4_mv_t(c, s, x, y, group=group, zeros=z)
        near_the_sum(y, x.double(), w, 16 + rows ** 0.5 / 2, f"{rows} x {cols} group {group} {vectors} vectors")


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("scales", TYPES)
def test_pack_with_zero_points_at_the_ends_of_the_range(name, scales):
    """Groups as wide as the type is (high - low is no fp32 number), larger than a scale can say, and so narrow that the scale is one of the smallest numbers of its type: 0 stays a
    value of its own, zero points are codes, and what no end of the range cuts off is off by half a step and the roundings of a quotient."""
    import torch
    most = 0.98 * float(torch.finfo(dtype(name)).max)      # (so that fifteen steps are a number where the scale is rounded up)
    smallest = TINY[scales]
    top = float(torch.finfo(dtype(scales)).max)
    rows = [(-0.9 * most, 0.9 * most), (-0.99 * most, 0.2 * most), (-0.1 * most, 0.95 * most), (-most, 0.0), (0.0, most)]
    rows += [(-21.0 * smallest, 0.0), (-22.0 * smallest, 0.5 * smallest), (-8.0 * smallest, 14.4 * smallest)] if scales == "f16" else []
    w = torch.empty(len(rows), 32, dtype=torch.float64)
    for r, (low, high) in enumerate(rows):
        w[r] = torch.linspace(low, high, 32, dtype=torch.float64)
        w[r, 5] = 0.0
    w = w.float().to(dtype(name))
    c = torch.empty(H.hbp_q4_shapes(len(rows), 32, 32)[0], dtype=torch.uint8, device="cuda")
    s = torch.empty(len(rows), 1, dtype=dtype(scales), device="cuda")
    z = torch.empty_like(s)
    H.hbp_q4_pack(w.cuda(), c, s, group=32, zeros=z)
    back = torch.from_numpy(values(c, s, z, 32, 32))
    assert torch.equal(H.hbp_q4_unpack(c, s, 32, group=32, zeros=z).cpu(), back.float())   # (half a step beyond the largest number is an infinity)
    s, z = s.cpu().double(), z.cpu().double()
    assert ((z >= 0) & (z <= 15) & (z == z.round())).all() and torch.isfinite(s).all() and not back[:, 5].any()
    wd = w.double()
    step = torch.stack([(wd[r].max().clamp(min=0) - wd[r].min().clamp(max=0)) / 15 for r in range(len(rows))])[:, None]
    assert ((s - step.clamp(max=top)).abs() <= UNIT[scales] * s * 1.001 + smallest / 2 + 2.0 ** -22 * s).all()
    inside = (wd / s + z >= 0) & (wd / s + z <= 15)
    assert inside[:, 5].all() and ((back - wd).abs()[inside] <= (s * (0.5 + 1e-5)).expand_as(wd)[inside]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("direction,vectors", [("mv", (1 << 21) + 70), ("mv_t", 262_141), ("mv_t", 327_691)])
def test_more_vectors_than_a_grid_has_passes(direction, vectors):
    import torch
    rows, cols = 3, 5
    c, s, z, w = matrix(rows, cols, 32, "f16", True, 3)
    n_in, n_out = (cols, rows) if direction == "mv" else (rows, cols)
    x = some_x(vectors, n_in, "bf16", 17)
    y = torch.full((vectors, n_out), float("nan"), dtype=x.dtype, device="cuda")
    print(f"[q4 vectors] {direction} {vectors}", flush=True)
    (H.hbp_q4_mv if direction == "mv" else H.hbp_q4_mv_t)(c, s, x.cuda(), y, group=32, zeros=z)
    agree(y, x.double().numpy() @ (w.T if direction == "mv" else w), x, "bf16")


def test_workspace_for_many_vectors_is_that_of_a_launch():
    need = [ctypes.c_size_t(), ctypes.c_size_t()]
    for n, vectors in zip(need, (1 << 20, 1 << 24)):
        assert H.lib().hbp_q4_mv_t_workspace(H.hbp_q4_matrix_t(4096, 4096, None, 64, 4096, 32, 0), vectors, n) == 0
    assert need[0].value == need[1].value < 4 << 30


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["f16", "bf16"])
@pytest.mark.parametrize("zeros", [False, True])
def test_products_of_16_bit_vectors_that_are_not_centred(name, zeros):
    """Codes on their way as 16 + q, against a sixteenth of what rounding x to 16 bits is worth: that much of the root of the terms' squares, beside the result's own rounding."""
    import torch
    for rows, cols, group, vectors in ((300, 4096, 128, 1), (300, 4096, 32, 4), (300, 4096, 512, 16), (8300, 2048, 64, 40), (66_000, 1000, 128, 2)):
        for kind, of in X_OF_ONE_SIGN.items():
            print(f"[q4 not centred] mv {rows} x {cols} group {group} zeros {zeros} {kind} {vectors} of {name}", flush=True)
            c, s, z, w = codes_around_their_zeros(rows, cols, group, "f32", zeros, group)
            x = of(torch.randn(vectors, cols, generator=torch.Generator(device="cuda").manual_seed(vectors), device="cuda")).to(dtype(name))
            y = torch.empty(vectors, rows, dtype=x.dtype, device="cuda")
            H.hbp_q4_mv(c, s, x, y, group=group, zeros=z)
            xd, wt = x.double(), w.t().contiguous()
            want, terms = torch.mm(xd, wt), torch.mm(xd.square(), wt.square()).sqrt()
            assert ((y.double() - want).abs() <= UNIT[name] * (want.abs() * (1 + 1e-6) + terms / 16)).all()
