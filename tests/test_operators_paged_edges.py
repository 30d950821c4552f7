"""Attention over a paged cache at the ends of what it takes: infinite values, long tails, large caps and scores, many long texts, large pages."""

import numpy as np
import pytest

import paper_2504_08860_amd as H
from test_operators_paged import INF, Batch, agree, cache_of
from test_operators_q4 import TINY, TYPES, UNIT, dtype


# Kernels: few rows, in pages of whole eights and of others; many rows, 128 and (a table with room for many positions) 256 a workgroup.
KERNELS = [dict(new=2, page=16), dict(new=2, page=5), dict(new=50, page=16), dict(new=200, page=16, kv_heads=2, wide=2048)]


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim", [8, 40, 64, 80, 96, 128, 136, 192, 256])
def test_infinite_values_that_all_rows_see(name, dim):
    """An infinite value in each eight positions of a step of 32 that some rows see more of, in columns of every quarter of a head: that column is infinite, all others are what they were."""
    import torch
    for how in KERNELS:
        new, page, kv_heads, wide = how["new"], how["page"], how.get("kv_heads", 1), how.get("wide", 0)
        b = Batch([(new, 94 + new)], name, kv_heads, 2, dim, page, seed=dim, wide=wide)     # (positions 64..93 are seen by all rows, 94 and 95 by some)
        want, off = b.reference()
        values = b.values.clone()
        for turn in range(4):
            columns = [(1, dim // 3, dim // 2 + 1, dim - 1)[(k + turn) % 4] for k in range(4)]
            signs = [INF, -INF, INF, -INF]
            (at, place) = b.slots(0, np.array([65, 73, 81, 89]))
            for k in range(4):
                b.values[int(at[k]), :, int(place[k]), columns[k]] = signs[k]
            print(f"[infinite values] {name} dim {dim} {how} turn {turn}", flush=True)
            got = b.attend()
            b.values.copy_(values)
            for k in range(4):
                assert (got[..., columns[k]] == signs[k]).all(), f"{how}: column {columns[k]}, eight {k}"
                got[..., columns[k]] = torch.from_numpy(want[..., columns[k]]).to(got)
            agree(got, want, off + UNIT[name] * np.abs(want), f"{how} turn {turn}")

@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
def test_scores_whose_differences_are_large(name):
    """Whole multiples of 2^10 to 2^100 as scores, exact in fp32, of which any two are equal or far apart: the result is the value at the largest one, or the mean of two values where there are two."""
    import torch
    rng = np.random.default_rng(7)
    # few rows, any page, 128 rows a workgroup, parts of both; 256 rows (a table with room for many positions) and wide heads
    for sizes, page, dim, kv_heads, wide in (([(3, 300), (1, 40)], 16, 64, 1, 0), ([(2, 300)], 5, 64, 1, 0), ([(50, 300)], 16, 64, 1, 0), ([(1, 9000)], 16, 64, 1, 0), ([(50, 9000)], 16, 64, 1, 0),
                                             ([(150, 300), (7, 100)], 16, 64, 4, 2048), ([(150, 300)], 16, 128, 4, 2048), ([(50, 300), (70, 9000)], 16, 256, 1, 0), ([(5, 300)], 16, 256, 1, 0)):
        for power in (10, 15, 16, 17, 18, 19, 20, 22, 26) if name == "f16" else (10, 18, 20, 26, 34, 60, 100):
            b = Batch(sizes, name, kv_heads, 2, dim, page, seed=power, wide=wide)
            # scores are n 2^power with whole numbers n up to 251, of 16 columns of queries times 16 of keys
            of_q = 2.0 ** min(power // 2 + 1, 14)
            of_k = 2.0 ** (power - 4) / of_q
            b.q[:], b.keys[:] = 0.0, 0.0
            b.q[..., :16] = of_q
            for scale in (1.0, -0.7, 0.3, 0.0517):
                for ties in (False, True):
                    tops = []
                    for s, (n, length) in enumerate(sizes):
                        numbers = rng.integers(0, 250, length)
                        tops.append(rng.choice(length - n + 1, 2 if ties else 1, replace=False))
                        numbers[tops[-1]] = 251
                        at, place = b.slots(s, np.arange(length))
                        b.keys[at, :, place, :16] = b.on(np.sign(scale) * numbers[:, None, None] * of_k).to(b.keys.dtype).expand(-1, kv_heads, 16)
                    assert torch.isfinite(b.keys).all()
                    print(f"[large scores] {name} {sizes} page {page} dim {dim} 2^{power} scale {scale} ties {ties}", flush=True)
                    got = b.attend(scale=scale).double().cpu().numpy()
                    for s, (n, length) in enumerate(sizes):
                        at, place = b.slots(s, tops[s])
                        v = b.values[at, :, place].double().cpu().numpy().repeat(2, 1)     # (of each query's head of keys)
                        # One weight times a value, or two equal ones: a 16-bit type's weights are rounded for the product and not for the sum, half a step; products, sums and their quotient are off
                        # by 8 roundings of fp32 at most, and the result is rounded once.
                        off = (8 * 2.0 ** -24 + (2 if name != "f32" else 1) * UNIT[name]) * np.abs(v).mean(0) + TINY[name]
                        rows = got[b.starts[s]:b.starts[s] + n]
                        assert (np.abs(rows - v.mean(0)) <= off).all(), f"{sizes} page {page} dim {dim} 2^{power} scale {scale} ties {ties}: {np.abs(rows - v.mean(0)).max()}"

@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("new,dim", [(1, 8), (40, 8), (300, 8), (40, 136)])
def test_one_position_that_outweighs_a_long_tail(name, new, dim):
    """One position with a score of 0 and 122879 of about -17.4: weights of 2^-25.1 of the largest one, which are 0.3 % of the sum together.  As many heads of keys as keep texts whole."""
    import torch
    size, times, heads = 4096, 30, 512
    length = size * times
    g = torch.Generator(device="cuda").manual_seed(new)
    keys, values = (torch.zeros(2, heads, size, dim, dtype=dtype(name), device="cuda") for _ in range(2))
    keys[..., 0] = -17.40625      # (as a number of the type, which is taken below)
    keys[0, :, 5, 0] = 0.0
    values.copy_(1 + 0.1 * torch.randn(values.shape, generator=g, device="cuda"))
    values[0, :, 5, :4] = 0.0
    q = torch.zeros(new, heads, dim, dtype=dtype(name), device="cuda")
    q[..., 0] = 1.0
    table = torch.tensor([[0] + [1] * (times - 1)], dtype=torch.int32, device="cuda")
    args = table, torch.tensor([0, new], dtype=torch.int32, device="cuda"), torch.tensor([length], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, float("nan"))
    H.hbp_paged_attention(q, keys, values, *args, out, scale=1.0)
    v, weight = values.double(), np.exp(float(keys[1, 0, 0, 0]))
    whole = v[0].sum(1) - v[0, :, 5] + (times - 2) * v[1].sum(1)
    for i in range(new):
        seen = size - new + i + 1      # of the last page
        tail, count = whole + v[1, :, :seen].sum(1), length - size + seen - 1
        sums = 1 + weight * count
        want = (v[0, :, 5] + weight * tail) / sums
        # Of scores with one term an exponent is off by 4 roundings of its size (25).  Weights of 16-bit types are off by half a step, and those of fp16, where they are small, by 2^-32 of the largest one
        # (which is held as 2^7 or more; 2^-25 is half the smallest step).  Sums of 122880 terms in fp32, of 8 lanes' and instructions' sums each: at most 15360 roundings, all of one sign, of half a step.
        most = UNIT[name] if name != "f32" else 0.0
        tiny = 2.0 ** -32 * tail / sums if name == "f16" else 0.0
        off = (most + (4 * 25 * 0.7 + 2 * 15360) * 2.0 ** -24) * want + tiny + UNIT[name] * want + TINY[name]
        worst = ((out[i].double() - want).abs() / off).max().item()
        assert worst <= 1, f"row {i}: {worst:.3g} times what is allowed"

@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
def test_caps_far_above_the_scores(name):
    """Caps of 10 to 10^30, and scores of a hundredth of the cap to three times it: what is lost in a capped score is relative to the score, not to the cap."""
    caps = (10.0, 4.0), (127.0, 4.0), (129.0, 4.0), (129.0, 30.0), (129.0, 100.0), (1e3, 5.0), (1e3, 600.0), (1e4, 5.0), (1e5, 5.0), (1e6, 5.0), (1e7, 5.0), (1e15, 5.0), (1e30, 5.0)
    few = (129.0, 100.0), (1e3, 600.0), (1e5, 5.0), (1e7, 5.0)
    for sizes, page, dim, kv_heads, wide, some in (([(2, 500), (1, 90)], 16, 128, 1, 0, caps), ([(2, 90)], 5, 128, 1, 0, caps), ([(50, 500)], 16, 128, 1, 0, caps), ([(60, 200)], 16, 40, 1, 0, few),
                                                   ([(100, 200)], 16, 64, 4, 2048, few), ([(100, 200)], 16, 96, 4, 2048, few), ([(40, 200)], 16, 256, 1, 0, few), ([(2, 200)], 16, 256, 1, 0, few)):
        for cap, spread in some:
            b = Batch(sizes, name, kv_heads, 2, dim, page, seed=int(cap) % 1000, wide=wide)
            b.q[:] = b.q * spread
            b.values[:] = b.values.abs()
            print(f"[caps] {name} {sizes} dim {dim} cap {cap} scores of {spread}", flush=True)
            got = b.attend(softcap=cap).double().cpu().numpy()
            q, keys, values = (t.double().cpu().numpy() for t in (b.q, b.keys, b.values))
            for s, (n, length) in enumerate(sizes):
                at, place = b.slots(s, np.arange(length))
                for h in range(kv_heads):
                    key, value = keys[at, h, place], values[at, h, place]
                    for i in range(n):
                        row, seen = q[b.starts[s] + i, 2 * h:2 * h + 2], length - n + i + 1
                        raw = row @ key[:seen].T * dim ** -0.5
                        terms = np.abs(row) @ np.abs(key[:seen]).T * dim ** -0.5
                        z = cap * np.tanh(raw / cap)
                        w = np.exp(z - z.max(1, keepdims=True))
                        w /= w.sum(1, keepdims=True)
                        # A score is off by 16 roundings of its terms (fp32: 64), which the cap does not make more of; tanh by 9 of its own size (worked through in fp32) and what it is of by 4, or, up to
                        # caps of 128, 4 of the cap; the exponent by 4 of its size.  A weight is off by what its score and the largest one are; 16-bit types' by half a step and fp16's by 2^-32.
                        z_off = 2.0 ** -24 * ((16 if name != "f32" else 64) * terms + 20 * np.abs(z) + (4 * cap if cap <= 128 and name != "f32" else 0.0) + 4)
                        w_off = 2 * z_off.max(1, keepdims=True) + 32 * 2.0 ** -24 + (UNIT[name] if name != "f32" else 0.0)
                        want = w @ value[:seen]
                        off = w_off * want + (2.0 ** -32 * value[:seen].sum(0) if name == "f16" else 0.0) + UNIT[name] * np.abs(want) + TINY[name]
                        worst = np.max(np.abs(got[b.starts[s] + i, 2 * h:2 * h + 2] - want) / off)
                        assert worst <= 1, f"{sizes} dim {dim} cap {cap} scores of {spread}: {worst:.3g} times what is allowed"

def test_scales_and_caps_that_32_bits_do_not_hold():
    """Refused before anything else is looked at, so also without rows."""
    def attend(scale, cap):
        return H.lib().hbp_paged_attention(cache_of(), 0, None, 0, 8, None, 0, scale, cap, 0, 1, None, 0, None)
    for scale, cap in ((3e38, 0.0), (-3e38, 0.0), (1.0, 3e38), (1.0, 2e30), (0.0, 3e38)):
        assert attend(scale, cap) == -1, (scale, cap)
    for scale, cap in ((1e38, 0.0), (1.0, 1e30), (0.0, 1e30), (1e-20, 1e10), (-0.1, 50.0)):
        assert attend(scale, cap) == 0, (scale, cap)

@pytest.mark.gpu
def test_many_long_texts():
    """256 texts of 129 times the same page of 65536 positions, 2^31 in all: as over the page once."""
    import torch
    n, size, dim, times = 256, 65536, 8, 129
    g = torch.Generator(device="cuda").manual_seed(0)
    r = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    keys, values, q = r(1, 1, size, dim).bfloat16(), (1 + 0.2 * r(1, 1, size, dim)).bfloat16(), r(n, 1, dim).bfloat16()
    table = torch.zeros(n, times, dtype=torch.int32, device="cuda")
    starts, lengths = torch.arange(n + 1, dtype=torch.int32, device="cuda"), torch.full((n,), size * times, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, float("nan"))
    H.hbp_paged_attention(q, keys, values, table, starts, lengths, out, most_new=1)
    z = q[:, 0].double() @ keys[0, 0].double().t().contiguous() * dim ** -0.5
    want = torch.softmax(z, 1) @ values[0, 0].double()
    assert not torch.isnan(out).any(), f"{int(torch.isnan(out).sum())} values were not written"
    # weights and the result are rounded to bf16, 2^-8 each at most; sums of 8 million terms over some thousand lanes, steps and parts are off by less than a thousandth of that
    assert ((out[:, 0].double() - want).abs() <= (2 * 2.0 ** -8 + 2.0 ** -10) * want.abs()).all()

def test_parts_and_places_for_them(tmp_path):
    """The rule by which texts are split, as the kernels have it, compiled for the CPU: never more parts than the host has counted on, for up to the most and the longest texts, and few heads of keys or many."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    (tmp_path / "split.cc").write_text(r"""
#include <stdio.h>
#include <stdlib.h>
#include "hbp_paged_split.h"
int main()
{
    unsigned long long state = 1;
    auto below = [&](double most) { state = state * 6364136223846793005ull + 1442695040888963407ull; return (long long)((state >> 11) / 9007199254740992.0 * most); };
    for (int i = 0; i < 200000; i++) {
        const int heads = 1 << below(17), wide = below(2);
        const int places = (wide ? 256 : 512) / heads > 1 ? (wide ? 256 : 512) / heads : 1, aim = (wide ? 512 : 1024) / heads > 1 ? (wide ? 512 : 1024) / heads : 1;
        const int enough = wide ? 2048 : 512, least = wide ? 256 : 128, whole = below(2) ? 512 : 1024, sequences = 1 + (int)below(40);
        const double longest = below(2) ? 2147418111.0 : 1 << below(31);     // 2^31 - 65537, the most
        long long total = 0, tiles_in_all = 0, units = 0, slots = 0;
        int spans[40], tiles[40];
        for (int s = 0; s < sequences; s++) {
            spans[s] = (int)(below(3) ? longest : below(longest + 1));
            tiles[s] = (int)below(below(2) ? 4 : 100000);
            total += (long long)spans[s] * tiles[s];
            tiles_in_all += tiles[s];
        }
        const int length = hbp::part_length((double)total, places, aim, enough, least);
        if (length < least || length % hbp::kStep) return printf("a length of %d\n", length), 1;
        for (int s = 0; s < sequences; s++) {
            const int parts = hbp::part_count(spans[s], length, whole);
            if (parts < 1) return printf("%d parts of %d positions\n", parts, spans[s]), 1;
            units += (long long)tiles[s] * parts;
            slots += parts > 1 ? (long long)tiles[s] * parts : 0;
        }
        if (units > tiles_in_all + aim + 1 || slots > 2 * aim + 2)
            return printf("%lld units of %lld tiles, %lld places for parts, aim %d, parts of %d positions\n", units, tiles_in_all, slots, aim, length), 1;
    }
    return 0;
}
""")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I" + os.path.join(root, "paper_2504_08860_amd", "csrc"), str(tmp_path / "split.cc"), "-o", str(tmp_path / "split")])
    subprocess.check_call([str(tmp_path / "split")])

@pytest.mark.gpu
@pytest.mark.parametrize("size", [65536, 65533])
def test_pages_of_more_than_2_31_positions_of_heads(size):
    """32800 heads of a page of 65536 positions: a page of 34 GB (keys and values are the same numbers in the same place), few rows and many."""
    import torch
    heads, dim = 32800, 8
    assert heads * size > 2 ** 31
    cache = torch.empty(1, heads, size, dim, dtype=torch.float16, device="cuda")
    table, starts, lengths = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([[0]], [0, 50], [50]))
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k = (torch.randn(50, heads, dim, generator=g, device="cuda").half() for _ in range(2))
    print(f"[large pages] {size}: append", flush=True)
    H.hbp_paged_append(k, k, cache, cache, table, starts, lengths)
    looked_at = [0, 1, 16400, 32767, 32768, 32799]
    for h in looked_at:
        assert torch.equal(cache[0, h, :50], k[:, h])
    out = torch.full_like(q, float("nan"))
    for new in (50, 1):
        print(f"[large pages] {size}: {new} rows", flush=True)
        starts[1] = new
        H.hbp_paged_attention(q[-new:], cache, cache, table, starts, lengths, out[-new:], most_new=new)
        assert torch.isfinite(out[-new:]).all()
        for h in looked_at:
            z = q[-new:, h].double() @ k[:, h].double().t().contiguous() * dim ** -0.5
            z = z.masked_fill(torch.arange(50, device="cuda") > torch.arange(50 - new, 50, device="cuda")[:, None], -INF)
            w = torch.softmax(z, 1)
            want, size_of = w @ k[:, h].double(), w @ k[:, h].double().abs()
            # weights are rounded to fp16 (half a step, or 2^-32 of the largest one) and the result; scores of 8 terms of up to 16, and sums of 50, are off by 2^-16 of a weight at the most
            assert ((out[-new:, h].double() - want).abs() <= (2.0 ** -11 + 2.0 ** -15) * size_of + 2.0 ** -11 * want.abs() + 2.0 ** -24).all(), (new, h)

@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
def test_rows_and_slots_beside_starts_that_are_none(name):
    """Starts that fall, lie below 0 or beyond the rows: rows of the other sequences are what they were, those of no sequence are left, in results and in the cache."""
    import torch
    # (starts, {rows that the attention computes: as with good starts}, {rows that are appended})
    for starts, good in (((0, 2, 99, 6), [0, 1]), ((-5, 2, 3, 6), [2, 3, 4, 5]), ((0, 2, 3, 7), [0, 1, 2]), ((0, 2, 3, 2 ** 31 - 1), [0, 1, 2]), ((-2 ** 31, 2, 3, 6), [2, 3, 4, 5])):
        b = Batch([(2, 40), (1, 9), (3, 50)], name, 1, 2, 64, 16)
        want, others = b.attend(), [i for i in range(6) if i not in good]
        places = [b.slots(s, np.arange(length - n, length)) for s, (n, length) in enumerate(b.sizes)]
        at, place = (np.concatenate(p) for p in zip(*places))
        b.args[1] = b.on(np.array(starts, np.int32))
        print(f"[starts that are none] {name} {starts}", flush=True)
        out = b.attend(out=torch.full_like(want, 7.0))
        assert bool(torch.equal(out[good], want[good])) and bool((out[others] == 7).all()), starts
        keys, values = b.keys.clone(), b.values.clone()
        keys[at[good], :, place[good]], values[at[good], :, place[good]] = b.k[good], b.v[good]
        H.hbp_paged_append(b.k, b.v, b.keys, b.values, *b.args)
        assert torch.equal(b.keys, keys) and torch.equal(b.values, values), starts
        q_out = torch.full_like(b.q, 7.0)
        H.hbp_paged_append(b.k, b.v, b.keys, b.values, *b.args, q=b.q, q_out=q_out)
        assert bool(torch.equal(q_out[good], b.q[good])) and bool((q_out[others] == 7).all()), starts
