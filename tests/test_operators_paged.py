"""A paged cache: new tokens appended with rotation, their attention over it, against numpy in 64 bits."""
import ctypes

import numpy as np
import pytest

import paper_2504_08860_amd as H
from test_operators_q4 import TINY, TYPES, UNIT, dtype

INF = float("inf")


class Batch:
    """Sequences with (new, cached with them) tokens, their pages in no order, rows of no sequence behind the last one; a cache of numbers."""

    def __init__(self, sizes, name, kv_heads=2, group=2, dim=64, page=16, seed=0, behind=0, spare=2, wide=0, apart=0, fill=None):
        import torch
        rng = self.rng = np.random.default_rng(seed)
        self.sizes, self.name, self.kv_heads, self.group, self.dim, self.page = sizes, name, kv_heads, group, dim, page
        self.starts = np.concatenate([[0], np.cumsum([n for n, _ in sizes])]).astype(np.int32)
        self.lengths = np.array([length for _, length in sizes], np.int32)
        self.tokens = int(self.starts[-1]) + behind
        used = [-(-max(length, 0) // page) for _, length in sizes]
        self.width = max([1] + used) + wide
        self.pages = sum(used) + spare
        order, at = rng.permutation(self.pages).astype(np.int32), 0
        self.table = np.full((len(sizes), self.width), -1, np.int32)
        for s, n in enumerate(used):
            self.table[s, :n] = order[at:at + n]
            at += n
        t = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype(name))  # noqa: E731
        both = t(self.pages, 2 + apart, kv_heads, page, dim) if fill is None else torch.full((self.pages, 2 + apart, kv_heads, page, dim), fill, dtype=dtype(name))
        both = both.cuda()
        self.keys, self.values = (both[:, 0], both[:, 1]) if apart else (both[:, 0].contiguous(), both[:, 1].contiguous())
        heads = kv_heads * group
        qkv = t(self.tokens, (heads + 2 * kv_heads) * dim)
        if apart:
            qkv = qkv.cuda()
        else:
            qkv = [p.contiguous().cuda() for p in qkv.split([heads * dim, kv_heads * dim, kv_heads * dim], 1)]
        if apart:
            qkv = qkv.split([heads * dim, kv_heads * dim, kv_heads * dim], 1)
        self.q, self.k, self.v = (p.view(self.tokens, -1, dim) for p in qkv)
        self.on = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
        self.args = [self.on(self.table), self.on(self.starts), self.on(self.lengths)]

    def write(self):
        """New tokens' keys and values into their slots, as they are."""
        H.hbp_paged_append(self.k, self.v, self.keys, self.values, *self.args)

    def slots(self, s, positions):
        """(page, place) of positions; page -1: not held"""
        which = np.asarray(positions) // self.page
        good = (which >= 0) & (which < self.width)
        page = np.where(good, self.table[s, np.where(good, which, 0)], -1)
        return np.where((page >= 0) & (page < self.pages), page, -1), np.asarray(positions) % self.page

    def attend(self, most_new=None, out=None, **how):
        import torch
        if out is None:
            out = torch.full_like(self.q.contiguous(), float("nan"))
        H.hbp_paged_attention(self.q, self.keys, self.values, *self.args, out, most_new=max([n for n, _ in self.sizes] + [1]) if most_new is None else most_new, **how)
        return out

    def reference(self, scale=None, softcap=0.0, window=0):
        """(results in 64 bits, what may be off), from the formula; rows of no sequence NaN"""
        scale = self.dim ** -0.5 if scale is None else scale
        q, keys, values = (t.double().cpu().numpy() for t in (self.q, self.keys, self.values))
        want, off = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
        for s, (n, length) in enumerate(self.sizes):
            j = np.arange(min(max(length, 0), self.width * self.page))
            page, place = self.slots(s, j)
            held = page >= 0
            for h in range(self.kv_heads):
                key, value = keys[np.maximum(page, 0), h, place], values[np.maximum(page, 0), h, place]
                for i in range(n):
                    p = length - n + i
                    sees = held & (j <= p) & ((j > p - window) if window else True)
                    heads = slice(h * self.group, (h + 1) * self.group)
                    row = q[self.starts[s] + i, heads]
                    if not sees.any():
                        want[self.starts[s] + i, heads], off[self.starts[s] + i, heads] = 0.0, 0.0
                        continue
                    z = row @ key[sees].T * scale
                    terms = (np.abs(row) @ np.abs(key[sees]).T * abs(scale)).max(1, keepdims=True)   # what a score's roundings are relative to
                    if softcap:
                        z = softcap * np.tanh(z / softcap)
                    w = np.exp(z - z.max(1, keepdims=True))
                    w /= w.sum(1, keepdims=True)
                    v = value[sees]
                    want[self.starts[s] + i, heads] = w @ v
                    # Roundings: of a score 16 of its terms (fp32: six products of parts, 2^-22 left out: 64), of an exponent as many of its size as its way has steps (with a cap 8 of that),
                    # of the weights (16-bit types) half a step each, of sums some; fp16 weights of less than 2^-14 of the largest one are off by 2^-25 of it.
                    steps = (16 if self.name != "f32" else 64) * (1 + terms) + 8 * softcap + 32
                    weights = UNIT[self.name] if self.name != "f32" else 0.0
                    tiny = 2.0 ** -25 * np.abs(v).sum(0) if self.name == "f16" else 0.0
                    off[self.starts[s] + i, heads] = (2 * steps * 2.0 ** -24 + weights) * (w @ np.abs(v)) + tiny
        return want, off + UNIT[self.name] * np.abs(want) + TINY[self.name]

    def check(self, what="", **how):
        got = self.attend(**how)
        how.pop("most_new", None)
        agree(got, *self.reference(**how), what)
        return got


def agree(got, want, off, what=""):
    got = got.double().cpu().numpy()
    rows = ~np.isnan(want)
    assert np.isnan(got[~rows]).all(), f"{what}: rows of no sequence were written"
    assert np.isfinite(got[rows]).all(), f"{what}: {np.argwhere(rows & ~np.isfinite(got))[:5].tolist()} not finite"
    worst = np.max(np.abs(got - want)[rows] / off[rows], initial=0.0)
    assert worst <= 1, f"{what}: {worst:.3g} times what is allowed, at {np.argwhere(rows & (np.abs(got - want) > off))[:5].tolist()}"


# ------------------------------------------------------------------------------------ appending

def rotated(x, positions, frequencies, interleaved):
    """(numpy in 64 bits, what may be off relative to roundings of fp32)"""
    x = x.double().cpu().numpy()
    out, size = x.copy(), np.zeros_like(x)
    pairs = len(frequencies)
    if pairs:
        angle = positions[:, None, None] * frequencies.astype(np.float64)
        a, b = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
        out[..., a] = x[..., a] * np.cos(angle) - x[..., b] * np.sin(angle)
        out[..., b] = x[..., b] * np.cos(angle) + x[..., a] * np.sin(angle)
        size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return out, size


def near(got, want, size, name, what):
    """Rounded once; the angle, in turns, is rounded to fp32 (3 roundings of a radian), sine and cosine, two products and a sum are off by some more: 16 in all."""
    got = got.double().cpu().numpy()
    off = UNIT[name] * np.abs(want) + 16 * 2.0 ** -24 * size + TINY[name]
    worst = np.max(np.abs(got - want) / off, initial=0.0)
    assert worst <= 1, f"{what}: {worst:.3g} times what is allowed"


def check_append(b, pairs, interleaved, with_queries=True, in_place=False):
    import torch
    frequencies = (10000.0 ** (-np.arange(pairs) / max(pairs, 1))).astype(np.float32)
    keys, values, q = b.keys.clone(), b.values.clone(), b.q.clone()
    q_out = None if not with_queries else b.q if in_place else torch.full_like(q.contiguous(), 7.0)
    H.hbp_paged_append(b.k, b.v, b.keys, b.values, *b.args, q=b.q if with_queries else None, q_out=q_out,
                       frequencies=b.on(frequencies) if pairs else None, interleaved=interleaved)
    want_k, want_v = keys.double().cpu().numpy(), values.double().cpu().numpy()
    size = np.zeros_like(want_k)
    for s, (n, length) in enumerate(b.sizes):
        rows = slice(b.starts[s], b.starts[s] + n)
        positions = length - n + np.arange(n)
        page, place = b.slots(s, positions)
        there = (page >= 0) & (positions >= 0)
        k, k_size = rotated(b.k[rows], positions, frequencies, interleaved)
        want_k[page[there], :, place[there]], size[page[there], :, place[there]] = k[there], k_size[there]
        want_v[page[there], :, place[there]] = b.v[rows].double().cpu().numpy()[there]
        if with_queries:
            near(q_out[rows], *rotated(q[rows], positions, frequencies, interleaved), b.name, "queries")
    near(b.keys, want_k, size, b.name, "keys")
    assert np.array_equal(b.values.double().cpu().numpy(), want_v)
    if with_queries:
        behind = slice(b.starts[-1], None)
        assert torch.equal(q_out[behind], q[behind] if in_place else torch.full_like(q[behind], 7.0))


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_append(name, interleaved):
    sizes = [(1, 1), (3, 40), (0, 17), (1, 100), (5, 5), (0, 0), (17, 61)]
    for k, (dim, pairs, page, kv_heads, group) in enumerate([(64, 32, 16, 2, 2), (128, 64, 64, 1, 7), (80, 16, 7, 3, 1), (8, 4, 1, 1, 1), (8, 0, 3, 2, 4), (24, 5, 16, 2, 3), (256, 128, 128, 1, 2),
                                                             (96, 44, 32, 5, 1), (128, 63, 48, 2, 9)]):
        print(f"[append] {name} dim {dim} pairs {pairs} page {page} heads {kv_heads} x {group}", flush=True)
        check_append(Batch(sizes, name, kv_heads, group, dim, page, seed=k, behind=k % 3, apart=k % 2, wide=k % 4), pairs, interleaved, with_queries=k != 3, in_place=k % 2 == 1)


@pytest.mark.gpu
def test_append_far_positions_and_slots_that_are_not_there():
    """Positions up to 2^31, angles of them (the last page is all that is held of such a text); positions below 0 and behind the table; pages that are none."""
    for length in (1_000_003, 2 ** 31 - 70000):
        b = Batch([(1, 1), (4, 30)], "f32", 1, 1, 16, 65536 if length > 2 ** 30 else 64)
        b.lengths[1] = length
        b.width = -(-length // b.page)
        b.sizes[1] = (4, length)
        b.table = np.full((2, b.width), -1, np.int32)
        b.table[0, 0], b.table[1, -1], b.table[1, -2] = 0, 1, 2
        b.args = [b.on(b.table), b.on(b.starts), b.on(b.lengths)]
        print(f"[append] {length} positions", flush=True)
        check_append(b, 8, False)
    for name in ("bf16", "f32"):
        b = Batch([(9, 4), (5, 50), (3, 3), (7, 20)], name, page=8, spare=3)   # nine tokens of a text of four: five before its beginning
        b.table[1, 6] = b.pages        # (positions 48, 49)
        b.table[3, 1] = -7
        b.lengths[2], b.sizes[2] = 8 * b.width + 2, (3, 8 * b.width + 2)   # the last two are behind the table
        b.args = [b.on(b.table), b.on(b.starts), b.on(b.lengths)]
        print(f"[append] slots that are not there, {name}", flush=True)
        check_append(b, 32, True)


# ------------------------------------------------------------------------------------ attention

@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim", [8, 40, 64, 80, 96, 128, 136, 192, 256])
def test_attention(name, dim):
    """One token to some, one position to some hundreds, rows that fill tiles and do not, pages of every kind."""
    for k, (sizes, kv_heads, group, page, how) in enumerate([
            ([(1, 1)], 1, 1, 16, {}),
            ([(1, 300), (1, 31), (1, 32), (1, 33), (0, 9), (1, 1000)], 2, 4, 16, {}),
            ([(3, 200), (16, 16), (1, 65), (7, 129)], 1, 5, 32, {"softcap": 5.0}),
            ([(33, 100), (2, 2), (70, 70)], 2, 1, 48, {"window": 40}),
            ([(5, 257), (40, 333), (1, 12)], 1, 8, 7, {"softcap": 20.0, "window": 33}),
            ([(20, 190), (1, 400)], 3, 3, 1, {"scale": -0.3}),
            ([(130, 400)], 1, 4, 128, {"window": 1})]):
        print(f"[attention] {name} dim {dim} case {k}", flush=True)
        Batch(sizes, name, kv_heads, group, dim, page, seed=dim + k, behind=k % 3, apart=k % 2, wide=k % 2, fill=None).check(f"case {k}", **how)


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
def test_attention_in_parts(name):
    """Long texts, which are split: alone, beside short ones, with windows, and many sequences."""
    for k, (sizes, kv_heads, group, dim, page, how) in enumerate([
            ([(1, 20_011)], 1, 4, 128, 16, {}),
            ([(3, 9000), (1, 5), (2, 700), (1, 12_345)], 2, 3, 64, 64, {"softcap": 30.0}),
            ([(5, 9000), (6, 4100)], 1, 2, 256, 32, {"window": 3000}),
            ([(1, 5000)], 1, 1, 96, 5, {}),
            ([(1 + i % 2, 1 + 37 * i % 500) for i in range(150)], 1, 2, 64, 16, {})]):
        print(f"[attention in parts] {name} case {k}", flush=True)
        Batch(sizes, name, kv_heads, group, dim, page, seed=k).check(f"case {k}", **how)


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim", [40, 64, 96, 128, 136])
def test_many_rows_of_long_tables(name, dim):
    """Tables with room for many positions, so that tiles are the largest ones: rows that fill them and do not, infinities and NaN behind texts and before windows, a page that
    is not held, and a new token's value that only later rows see."""
    import torch
    for k, (sizes, kv_heads, group, page, how) in enumerate([
            ([(150, 700), (0, 5), (65, 65), (257, 900), (1, 333)], 1, 2, 16, {}),
            ([(100, 160), (90, 1300), (3, 50)], 2, 4, 64, {"softcap": 20.0}),
            ([(200, 600), (129, 129)], 52, 3, 8, {"window": 75})]):
        print(f"[long tables] {name} dim {dim} case {k}", flush=True)
        b = Batch(sizes, name, kv_heads, group, dim, page, seed=dim + k, wide=32768 // page)
        if k == 0:
            b.table[0, 3] = -1
            b.args[0] = b.on(b.table)
        want = b.check(f"case {k}", **how)
        window, unseen = how.get("window", 0), torch.ones(b.pages, page, dtype=torch.bool)
        for s, (n, length) in enumerate(sizes):
            at, place = b.slots(s, np.arange(max(0, length - n - window + 1) if window else 0, length))
            unseen[at[at >= 0], place[at >= 0]] = False
        for bad in (float("nan"), INF):
            keys, values = b.keys.clone(), b.values.clone()
            b.keys.masked_fill_(unseen.cuda()[:, None, :, None], bad)
            b.values.masked_fill_(unseen.cuda()[:, None, :, None], bad)
            n, length = sizes[0]
            (at,), (place,) = b.slots(0, np.array([length - 9]))
            b.values[at, :, place, 5] = bad
            got = b.attend(**how)
            rows = np.ones(b.tokens, bool)
            rows[n - 9:n] = False
            assert torch.equal(got[rows], want[rows])
            assert not torch.isfinite(got[~rows][:, :, 5]).any()
            others = np.arange(dim) != 5
            assert torch.equal(got[~rows][:, :, others], want[~rows][:, :, others])
            b.keys.copy_(keys), b.values.copy_(values)


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("page", [16, 5])
def test_what_a_query_does_not_see(name, page):
    """NaN and infinities in slots behind a text, in pages of no one, before a window, and in new tokens that only later rows see."""
    import torch
    for window in (0, 20):
        for bad in (float("nan"), INF, -INF):
            b = Batch([(6, 100), (1, 45), (40, 40), (9, 75)], name, 2, 2, 64, page, seed=3, fill=None)
            held = torch.zeros(b.pages, page, dtype=torch.bool)
            for s, (n, length) in enumerate(b.sizes):
                at, place = b.slots(s, np.arange(max(0, length - n - window + 1) if window else 0, length))
                held[at, place] = True
            gone = ~held.cuda()
            b.keys.masked_fill_(gone[:, None, :, None], bad)
            b.values.masked_fill_(gone[:, None, :, None], bad)
            print(f"[unseen] {name} page {page} window {window} {bad}", flush=True)
            want = b.check("unseen slots", window=window)
            # a new token of the first and the third sequence: rows before it are as they were
            for s, at in ((0, 97), (2, 33)):
                (page_at,), (place,) = b.slots(s, np.array([at]))
                b.keys[page_at, :, place, 3], b.values[page_at, :, place, 5] = bad, bad
            got = b.attend(window=window)
            rows = np.ones(b.tokens, bool)
            rows[3:6] = rows[7 + 33:7 + 40] = False
            assert torch.equal(got[rows], want[rows])
            if not bad < 0:
                assert not torch.isfinite(got[~rows][:, :, 5]).any()
            assert torch.isnan(got[~rows]).any() or bad < 0


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
def test_pages_that_are_not_held_and_rows_that_see_nothing(name):
    import torch
    for page in (8, 12):
        b = Batch([(3, 64), (2, 50), (4, 3), (1, 40), (2, 30)], name, 1, 3, 64, page, seed=1)
        b.table[0, 2:4] = -1
        b.table[1, 1] = b.pages
        b.table[3, :] = -1       # nothing at all
        b.lengths[4], b.sizes[4] = b.width * page + 2, (2, b.width * page + 2)   # two rows behind the table see what is in it
        b.table[4] = b.table[0, 0]
        b.args = [b.on(b.table), b.on(b.starts), b.on(b.lengths)]
        print(f"[attention] pages that are not held, {name} {page}", flush=True)
        b.check("holes")
        b.check("holes, window", window=9)
    b = Batch([(2, 40)], name, 1, 2, 64, 16)
    b.keys.fill_(-INF if name != "f32" else -3e38)   # scores of -inf alone: 0, too
    b.q.fill_(1.0 if name != "f32" else 3e38)
    assert (b.attend() == 0).all()
    out = torch.full_like(b.q, 5.0)
    H.hbp_paged_attention(b.q, b.keys, b.values, *b.args, out, most_new=1)   # (rows behind most_new stay as they are)
    assert (out[:1] == 0).all() and (out[1:] == 5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
def test_attention_of_extreme_scores(name):
    """Scores far from zero, growing and falling along the text; one position that outweighs all others, first and last."""
    for dim, page in ((64, 16), (128, 64)):
        b = Batch([(2, 700), (1, 333)], name, 1, 2, dim, page, seed=9)
        for size in (1e-3, 8.0):
            for ramp in (0.0, 0.2, -0.2):
                b.q[:] = size
                for s, (n, length) in enumerate(b.sizes):
                    at, place = b.slots(s, np.arange(length))
                    b.keys[at, 0, place] = b.on(np.repeat((ramp * np.arange(length))[:, None], dim, 1)).to(b.keys.dtype) + b.keys[at, 0, place] * 0.1
                print(f"[attention] scores {size} x {ramp} {name} dim {dim}", flush=True)
                b.check(f"{size} {ramp}")


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
def test_queries_that_are_no_numbers(name):
    """NaN and infinities in one row's query are that row's alone."""
    import torch
    for sizes, page in (([(3, 300), (1, 40)], 16), ([(3, 300), (1, 40)], 5), ([(50, 300), (1, 40)], 16)):
        b = Batch(sizes, name, 1, 2, 64, page, seed=2)
        want = b.attend()
        b.q[1, 0, 5], b.q[2, 1, 7] = float("nan"), INF
        got = b.attend()
        rows = [i for i in range(b.tokens) if i not in (1, 2)]
        assert torch.equal(got[rows], want[rows]) and torch.equal(got[1, 1], want[1, 1]) and torch.equal(got[2, 0], want[2, 0])
        assert torch.isnan(got[1, 0]).all() and torch.isnan(got[2, 1]).all()


@pytest.mark.gpu
def test_infinite_visible_values_of_fp32():
    """Infinities that a row does see: scores of -inf have no weight, infinite values give infinities."""
    import torch
    b = Batch([(2, 50)], "f32", 1, 1, 64, 16, seed=4)
    b.q[:] = b.q.abs()
    (page, _), (place, _) = b.slots(0, np.array([10, 11]))
    b.keys[page, 0, place] = -INF
    got = b.attend()
    keep = b.keys[page, 0, place].clone()
    b.keys[page, 0, place] = -1e30       # (as good as -inf: no weight either)
    want = b.attend()
    assert torch.equal(got, want) and torch.isfinite(got).all()
    b.keys[page, 0, place] = keep
    b.values[page, 0, place + 1, 7] = INF
    got = b.attend()
    assert (got[:, 0, 7] == INF).all()
    # The other columns are summed in another way: either sum has 50 terms w v with weights that add up to 1, at most 52 roundings and 2^-22 from products of parts, each relative to the
    # largest |v|: 56 * 2^-24 of it either way.
    assert (got[:, 0, :7] - want[:, 0, :7]).abs().max() <= 2 * 56 * 2.0 ** -24 * b.values[torch.isfinite(b.values)].abs().max()


@pytest.mark.gpu
def test_in_place_streams_and_graphs():
    """Queries' own memory for results; another stream; a captured step that is replayed with other lengths, tables and tokens."""
    import torch
    b = Batch([(2, 5000), (1, 70), (3, 900)], "bf16", 2, 4, 128, 16, seed=5)
    want = b.attend(softcap=30.0)
    b2 = b.q.clone()
    H.hbp_paged_attention(b2, b.keys, b.values, *b.args, b2, softcap=30.0, most_new=3)
    assert torch.equal(want, b2)
    side = torch.cuda.Stream()
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    H.hbp_paged_attention(b.q, b.keys, b.values, *b.args, out, softcap=30.0, most_new=3, stream=side)
    side.synchronize()
    assert torch.equal(want, out)

    frequencies = torch.rand(64, device="cuda")
    q_out, out = torch.empty_like(b.q), torch.empty_like(b.q)

    def step():
        H.hbp_paged_append(b.k, b.v, b.keys, b.values, *b.args, q=b.q, q_out=q_out, frequencies=frequencies)
        H.hbp_paged_attention(q_out, b.keys, b.values, *b.args, out, most_new=3)
    keys, values = b.keys.clone(), b.values.clone()
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lengths in ((5000, 70, 900), (4000, 1, 3), (4999, 80, 33), (2, 3, 4)):
        b.args[2].copy_(torch.tensor(lengths, dtype=torch.int32))
        b.q.normal_(), b.k.normal_()
        results = []
        for go in (step, graph.replay):
            b.keys.copy_(keys), b.values.copy_(values)
            out.fill_(float("nan"))
            torch.cuda.synchronize()
            go()
            torch.cuda.synchronize()
            results.append((out.clone(), q_out.clone(), b.keys.clone(), b.values.clone()))
        assert all(torch.equal(x, y) for x, y in zip(*results)) and torch.isfinite(results[0][0]).all()


@pytest.mark.gpu
def test_two_graphs_at_once():
    """Two captured steps on two streams, each with a workspace of its own."""
    import torch
    batches = [Batch([(1, 9000 + 100 * i), (2, 400)], "f16", 1, 4, 128, 16, seed=i) for i in range(2)]
    wants = [b.attend() for b in batches]
    outs, graphs, streams = [torch.empty_like(w) for w in wants], [], [torch.cuda.Stream() for _ in batches]
    for b, out in zip(batches, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            H.hbp_paged_attention(b.q, b.keys, b.values, *b.args, out, most_new=2)
        graphs.append(g)
    for _ in range(20):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(w, o) for w, o in zip(wants, outs))


@pytest.mark.gpu
@pytest.mark.parametrize("page", [16, 5])
def test_pages_further_apart_than_32_bits_count(page):
    import torch
    b = Batch([(3, 900)], "bf16", 2, 2, 128, page, seed=6)
    apart = (5 << 30) // b.pages // 8 * 8     # 10 GB in all
    far = torch.empty(b.pages * apart, dtype=torch.bfloat16, device="cuda")
    size = 2 * page * 128
    view = lambda at: far.as_strided((b.pages, 2, page, 128), (apart, page * 128, 128, 1), at)  # noqa: E731
    keys, values = view(0), view(size)
    keys.copy_(b.keys), values.copy_(b.values)
    near_by = b.attend()
    k, v = b.k.clone(), b.v.clone()
    H.hbp_paged_append(k, v, keys, values, *b.args)
    b.write()
    assert torch.equal(keys, b.keys) and torch.equal(values, b.values)
    want = b.attend()
    b.keys, b.values = keys, values
    assert torch.equal(b.attend(), want) and not torch.equal(near_by, want)


@pytest.mark.gpu
def test_many_sequences():
    """Thousands of sequences, against the same ones some at a time."""
    import torch
    sizes = [(1 + i % 3 if i % 11 else 0, 3 + 17 * i % 260) for i in range(5000)]
    b = Batch(sizes, "f16", 1, 2, 64, 16, seed=8)
    got = b.attend()
    keys, values, args = b.keys.clone(), b.values.clone(), b.args
    for a, z in ((0, 60), (2000, 2070), (4935, 5000)):
        out = torch.empty_like(b.q[b.starts[a]:b.starts[z]])
        H.hbp_paged_attention(b.q[b.starts[a]:b.starts[z]], keys, values, args[0][a:z], args[1][a:z + 1] - args[1][a], args[2][a:z], out, most_new=3)
        assert (got[b.starts[a]:b.starts[z]].float() - out.float()).abs().max() <= 4 * UNIT["f16"] * out.float().abs().max()   # (other parts: other roundings)
    b.write()
    for s in (0, 1, 2500, 4999):
        n, length = sizes[s]
        at, place = b.slots(s, np.arange(length - n, length))
        assert torch.equal(b.keys[at, :, place], b.k[b.starts[s]:b.starts[s + 1]])


def test_divisions_by_page_sizes_and_groups():
    """The rule that positions are divided by, in numpy: the quotient for every divisor up to 70000 and some beyond, at multiples and beside them."""
    for d in list(range(1, 3000)) + [4096, 65535, 65536, 70000, 2 ** 30 + 1, 2 ** 31 - 1]:
        s = max(0, (d - 1).bit_length())
        m = -(-(1 << (31 + s)) // d)
        assert m < 1 << 32
        for n in {0, 1, d - 1, d, d + 1, 2 ** 31 - 1, (2 ** 31 - 1) // d * d, max(0, (2 ** 31 - 1) // d * d - 1)}:
            if n < 2 ** 31:
                assert n * m >> (31 + s) == n // d


# ------------------------------------------------------------------------------------ refusals

def cache_of(**change):
    good = dict(keys=4096, values=4096, table=4096, starts=4096, lengths=4096, ldk=2048, ldv=2048, ldt=4, pages=8, sequences=2, table_width=4, type=1, kv_heads=2,
                page_size=16, head_dim=64)
    return H.hbp_paged_t(*[(good | change)[k] for k, _ in H.hbp_paged_t._fields_])


BAD_CACHES = [dict(keys=None), dict(values=None), dict(keys=4104), dict(values=4098), dict(table=None), dict(table=4098), dict(starts=None), dict(starts=4097), dict(lengths=None),
              dict(ldk=2040), dict(ldv=2047), dict(ldk=2052), dict(ldt=3), dict(pages=0), dict(sequences=-1), dict(table_width=0), dict(type=5), dict(kv_heads=0),
              dict(page_size=0), dict(head_dim=0), dict(head_dim=60), dict(head_dim=264)]
LARGE_CACHES = [dict(pages=1 << 31), dict(pages=1 << 27), dict(page_size=70000, ldk=1 << 40, ldv=1 << 40), dict(sequences=1 << 25)]


def test_what_the_library_refuses():
    L = H.lib()

    def append(cache=None, tokens=3, k=4096, ldk=128, v=4096, ldv=128, q=4096, ldq=512, heads=8, qo=4096, ldqo=512, f=4096, pairs=32):
        return L.hbp_paged_append(cache or cache_of(), tokens, k, ldk, v, ldv, q, ldq, heads, qo, ldqo, f, pairs, 0, None)

    def attend(cache=None, tokens=3, q=4096, ldq=512, heads=8, out=4096, ldo=512, scale=1.0, cap=0.0, window=0, most=1, ws=4096, size=1 << 40):
        return L.hbp_paged_attention(cache or cache_of(), tokens, q, ldq, heads, out, ldo, scale, cap, window, most, ws, size, None)
    for call in (append, attend):
        for bad in BAD_CACHES:
            assert call(cache_of(**bad)) == -1, bad
        for large in LARGE_CACHES:
            assert call(cache_of(**large)) == -4, large
        assert call(tokens=-1) == -1 and call(tokens=0) == 0 and call(cache_of(sequences=0)) == 0
    for bad in (dict(k=None), dict(k=4097), dict(v=None), dict(v=4097), dict(ldk=127), dict(ldv=1), dict(q=None), dict(qo=None), dict(heads=0), dict(heads=-1), dict(ldq=511),
                dict(ldqo=511), dict(f=None), dict(f=4098), dict(pairs=-1), dict(pairs=33), dict(q=4097), dict(qo=4099)):
        assert append(**bad) == -1, bad
    assert append(tokens=(1 << 30) + 1) == -4
    nan = float("nan")
    for bad in (dict(q=None), dict(q=4097), dict(out=None), dict(out=4097), dict(ldq=511), dict(ldo=511), dict(heads=0), dict(heads=7), dict(scale=nan), dict(scale=INF), dict(cap=-1.0),
                dict(cap=nan), dict(cap=INF), dict(cap=1e-44), dict(window=-1), dict(most=-1)):
        assert attend(**bad) == -1, bad
    assert attend(tokens=1 << 30) == -4 and attend(most=0) == 0
    need, long = ctypes.c_size_t(), cache_of(pages=1 << 20, table_width=1 << 19, ldt=1 << 19)
    assert L.hbp_paged_attention_workspace(long, 3, 8, 0, 1, need) == 0 and need.value > 0
    for ws, size in ((None, need.value), (4096, need.value - 1), (4100, need.value)):
        assert attend(long, ws=ws, size=size) == -1
    assert L.hbp_paged_attention_workspace(long, 3, 8, 0, 1, None) == -1 and L.hbp_paged_attention_workspace(long, 3, 7, 0, 1, need) == -1
    assert L.hbp_paged_attention_workspace(None, 3, 8, 0, 1, need) == -1
    assert L.hbp_paged_attention_workspace(cache_of(), 3, 8, 0, 1, need) == 0 and need.value == 0     # (64 positions are not split)


def test_struct_of_the_cache_matches_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    fields = [f for f, _ in H.hbp_paged_t._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hbp.h"\nint main(void){printf("%zu\\n", sizeof(hbp_paged_t));'
                   + "".join(f'printf("%zu\\n", offsetof(hbp_paged_t, {f}));' for f in fields) + "return 0;}")
    subprocess.check_call(["gcc", "-I" + os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "layout")]).split()]
    assert got == [ctypes.sizeof(H.hbp_paged_t)] + [getattr(H.hbp_paged_t, f).offset for f in fields]


@pytest.mark.gpu
def test_what_the_binding_refuses():
    import torch
    b = Batch([(2, 40), (1, 9)], "f16", 2, 2, 64, 16)
    table, starts, lengths = b.args
    out, q_out, f = torch.empty_like(b.q), torch.empty_like(b.q), torch.ones(32, device="cuda")
    good = dict(k=b.k, v=b.v, keys=b.keys, values=b.values, table=table, starts=starts, lengths=lengths, q=b.q, q_out=q_out, frequencies=f)
    caches = [dict(keys=b.keys.float()), dict(keys=b.keys[0]), dict(keys=b.keys.cpu()), dict(values=b.values[:-1]), dict(values=b.values.transpose(1, 2)), dict(keys=b.keys[..., ::2]),
              dict(table=table[0]), dict(table=table.long()), dict(table=table.t()), dict(starts=starts[:-1]), dict(starts=starts.long()), dict(lengths=lengths[:1]), dict(lengths=lengths.cpu())]
    for change in caches + [dict(k=b.k[:1]), dict(k=b.k[:, :1]), dict(v=b.v.float()), dict(v=b.v[..., :32]), dict(q=None), dict(q_out=None), dict(q=b.q[0]), dict(q=b.q[:2]),
                            dict(q_out=q_out[:, :2]), dict(frequencies=f.double()), dict(frequencies=f[::2]), dict(frequencies=f[None])]:
        with pytest.raises(AssertionError):
            H.hbp_paged_append(**good | change)
    with pytest.raises(H.HbpError):
        H.hbp_paged_append(**good | dict(frequencies=torch.ones(33, device="cuda")))
    good = dict(q=b.q, keys=b.keys, values=b.values, table=table, starts=starts, lengths=lengths, out=out)
    for change in caches + [dict(q=b.q[0]), dict(q=b.q.float()), dict(q=b.q[..., :32]), dict(out=out[:2]), dict(out=out.transpose(0, 1)), dict(out=out.cpu())]:
        with pytest.raises(AssertionError):
            H.hbp_paged_attention(**good | change)
    for change in (dict(window=-1), dict(softcap=-1.0), dict(scale=float("nan")), dict(q=b.q[:, :3], out=out[:, :3].contiguous())):
        with pytest.raises(H.HbpError):
            H.hbp_paged_attention(**good | change)
    none = torch.empty(0, 4, 64, dtype=torch.float16, device="cuda")
    H.hbp_paged_attention(none, b.keys, b.values, table, starts * 0, lengths, none)
    H.hbp_paged_append(none[:, :2], none[:, :2], b.keys, b.values, table, starts * 0, lengths)


@pytest.mark.gpu
def test_starts_that_are_none():
    """Starts that fall, lie below 0 or beyond the rows: such sequences have no rows, the others theirs."""
    import torch
    b = Batch([(2, 40), (1, 9), (3, 50)], "bf16", 1, 2, 64, 16)
    want = b.attend()
    for starts, good in (((0, 2, 99, 6), [0, 1]), ((-5, 2, 3, 6), [2, 3, 4, 5]), ((0, 2, 1, 6), [0])):
        b.args[1] = b.on(np.array(starts, np.int32))
        keys, values = b.keys.clone(), b.values.clone()
        out = b.attend(out=torch.zeros_like(want))
        assert all(torch.equal(out[i], want[i]) for i in good[:1])
        H.hbp_paged_append(b.k, b.v, b.keys, b.values, *b.args)
        b.keys.copy_(keys), b.values.copy_(values)
