// New tokens' keys and values into a paged cache, keys and queries rotated by their positions on the way (hbp_paged_append).
#include "hbp_paged.h"

#include <algorithm>

namespace hbp {
namespace {

struct AppendArgs {
    Paged c;
    const void *k, *v, *q;
    void *q_out;
    int64_t ldk, ldv, ldq, ldqo;
    const float *frequencies;
    int32_t tokens, heads, pairs, interleaved;
    Divider by_rotated, by_copied;   // units of a head of keys or queries, and of values
};

// U values at an address of which only the value's own alignment is known
template <typename T, int U> struct Values {
    T v[U];
    struct __attribute__((packed, aligned(sizeof(T)))) raw_t { T v[U]; };
    __device__ __forceinline__ void load(const T *p)
    {
        const raw_t r = *reinterpret_cast<const raw_t *>(p);
#pragma unroll
        for (int i = 0; i < U; i++) v[i] = r.v[i];
    }
    __device__ __forceinline__ void store(T *p) const
    {
        raw_t r;
#pragma unroll
        for (int i = 0; i < U; i++) r.v[i] = v[i];
        *reinterpret_cast<raw_t *>(p) = r;
    }
};

// One workgroup a token at a time.  The token's cosines and sines are made once, for all heads, in LDS.  A thread's unit is U pairs of a head of keys or queries (both values of
// a pair in one thread, so that queries may be rotated in place), U values behind the rotated ones, or U values of a head of values.  The first kAhead units are loaded before the
// position is known.  Bound: HBM; 10000 tokens of 40 + 8 + 8 heads of 80 fp32 values 71 us, 4.2 TB/s read and written; one token of 32 + 8 + 8 heads of 128 2.4 us, a chain of loads.
constexpr int kThreads = 256, kAhead = 2;
template <typename T, int U> __global__ __launch_bounds__(kThreads) void k_paged_append(AppendArgs a)
{
    __shared__ float2 turns[128];
    const int32_t rotated = a.by_rotated.d, copied = a.by_copied.d, dim = a.c.head_dim, turning = a.pairs / U;
    const int32_t rotated_units = (a.heads + a.c.kv_heads) * rotated, units = rotated_units + a.c.kv_heads * copied;
    for (int32_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        Values<T, U> x[kAhead], y[kAhead];
        // where a unit's two halves are: the head (queries, then keys, then values), and offsets in it (second < 0: none)
        auto place = [&](int32_t unit, int32_t &head, int32_t &first, int32_t &second, int32_t &pair) {
            if (unit < rotated_units) {
                head = a.by_rotated.divide(unit);
                const int32_t k = unit - head * rotated;
                pair = k * U;
                first = a.interleaved ? 2 * pair : pair;
                second = a.interleaved ? first + U : pair + a.pairs;
                if (k >= turning) {
                    first = 2 * a.pairs + (k - turning) * U;
                    second = -1;
                }
            } else {
                const int32_t k = unit - rotated_units;
                head = a.by_copied.divide(k);
                first = (k - head * copied) * U;
                second = -1;
                pair = 0;
                head += a.heads + a.c.kv_heads;
            }
        };
        auto source = [&](int32_t head) -> const T * {
            if (head < a.heads) return static_cast<const T *>(a.q) + t * a.ldq + (int64_t)head * dim;
            head -= a.heads;
            if (head < a.c.kv_heads) return static_cast<const T *>(a.k) + t * a.ldk + (int64_t)head * dim;
            return static_cast<const T *>(a.v) + t * a.ldv + (int64_t)(head - a.c.kv_heads) * dim;
        };
        auto load = [&](int32_t from) {
#pragma unroll
            for (int i = 0; i < kAhead; i++) {
                const int32_t unit = from + i * kThreads + threadIdx.x;
                if (unit >= units) continue;
                int32_t head, first, second, pair;
                place(unit, head, first, second, pair);
                const T *at = source(head);
                x[i].load(at + first);
                if (second >= 0) y[i].load(at + second);
            }
        };
        load(0);
        const int32_t s = sequence_of(a.c.starts, a.c.sequences, t);
        if (s >= a.c.sequences) continue;   // (the same in all threads)
        const int32_t begin = a.c.starts[s], end = a.c.starts[s + 1];
        if (begin < 0 || begin > t || end > a.tokens) continue;   // (of no sequence, or of one whose rows are not all there, as in the attention)
        const int64_t position = (int64_t)a.c.lengths[s] - (end - t);
        int64_t page = -1, within = 0;
        if (position >= 0 && position < a.c.capacity) {
            const int32_t which = a.c.by_page.divide((int32_t)position);
            page = a.c.table[s * a.c.ldt + which];
            if (page >= a.c.pages) page = -1;
            within = (position - (int64_t)which * a.c.page_size) * dim;
        }
        if ((int)threadIdx.x < a.pairs) {
            // the angle as a part of a turn: of 2^31 positions times a frequency of 1 turn, 64 bits leave 2^-22 of a turn, and 2^-33 of a position below a million
            constexpr double kTurns = 0.15915494309189533577;   // 1 / (2 pi)
            const double turn = (double)position * (double)a.frequencies[threadIdx.x] * kTurns;
            float sine, cosine;
            sincospif(2.0f * (float)(turn - rint(turn)), &sine, &cosine);
            turns[threadIdx.x] = float2{cosine, sine};
        }
        __syncthreads();
        for (int32_t from = 0; from < units; from += kAhead * kThreads) {
            if (from) load(from);
#pragma unroll
            for (int i = 0; i < kAhead; i++) {
                const int32_t unit = from + i * kThreads + threadIdx.x;
                if (unit >= units) continue;
                int32_t head, first, second, pair;
                place(unit, head, first, second, pair);
                if (second >= 0) {
                    Values<T, U> f = x[i], g = y[i];
                    if (a.interleaved) {
                        // (2U values in a row: pairs lie side by side)
#pragma unroll
                        for (int j = 0; j < U; j++) {
                            const float2 turn = turns[pair + j];
                            auto value = [&](int at) { return to_f32(at < U ? x[i].v[at < U ? at : 0] : y[i].v[at < U ? 0 : at - U]); };
                            const float even = value(2 * j), odd = value(2 * j + 1);
                            const T re = from_f32<T>(even * turn.x - odd * turn.y), im = from_f32<T>(odd * turn.x + even * turn.y);
                            if (2 * j < U) f.v[2 * j < U ? 2 * j : 0] = re; else g.v[2 * j < U ? 0 : 2 * j - U] = re;
                            if (2 * j + 1 < U) f.v[2 * j + 1 < U ? 2 * j + 1 : 0] = im; else g.v[2 * j + 1 < U ? 0 : 2 * j + 1 - U] = im;
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < U; j++) {
                            const float2 turn = turns[pair + j];
                            const float re = to_f32(x[i].v[j]), im = to_f32(y[i].v[j]);
                            f.v[j] = from_f32<T>(re * turn.x - im * turn.y);
                            g.v[j] = from_f32<T>(im * turn.x + re * turn.y);
                        }
                    }
                    x[i] = f;
                    y[i] = g;
                }
                T *to;
                if (head < a.heads) {
                    to = static_cast<T *>(a.q_out) + t * a.ldqo + (int64_t)head * dim;
                } else {
                    if (page < 0) continue;
                    const bool value = head >= a.heads + a.c.kv_heads;
                    const int64_t of_head = (int64_t)(head - a.heads - (value ? a.c.kv_heads : 0)) * a.c.page_size * dim + within;
                    to = value ? static_cast<T *>(const_cast<void *>(a.c.values)) + page * a.c.ldv + of_head
                               : static_cast<T *>(const_cast<void *>(a.c.keys)) + page * a.c.ldk + of_head;
                }
                x[i].store(to + first);
                if (second >= 0) y[i].store(to + second);
            }
        }
        __syncthreads();   // (before the next token's turns)
    }
}

}  // namespace
}  // namespace hbp

extern "C" int hbp_paged_append(const hbp_paged_t *cache, int64_t tokens, const void *k, int64_t ldk, const void *v, int64_t ldv, const void *q, int64_t ldq,
                                int heads, void *q_out, int64_t ldqo, const float *frequencies, int pairs, int interleaved, void *stream)
{
    using namespace hbp;
    AppendArgs a{};
    int rc = check_paged(cache, &a.c);
    if (rc != HBP_OK) return rc;
    if (tokens < 0 || heads < 0 || pairs < 0 || 2 * (int64_t)pairs > cache->head_dim || (pairs && !frequencies) || !aligned(frequencies, 4)) return HBP_ERR_INVALID_ARGUMENT;
    if (tokens > (int64_t(1) << 30) || heads > 65536) return HBP_ERR_TOO_LARGE;
    if (tokens == 0 || cache->sequences == 0) return HBP_OK;
    const int64_t bytes = type_bytes(cache->type), dim = cache->head_dim, kv = cache->kv_heads * dim;
    if (!k || !v || !aligned(k, bytes) || !aligned(v, bytes) || (heads > 0) != (q != nullptr) || (heads > 0) != (q_out != nullptr) || !aligned(q, bytes) ||
        !aligned(q_out, bytes)) return HBP_ERR_INVALID_ARGUMENT;
    if (tokens > 1 && (ldk < kv || ldv < kv || (heads && (ldq < heads * dim || ldqo < heads * dim)))) return HBP_ERR_INVALID_ARGUMENT;
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    a.k = k; a.v = v; a.q = q; a.q_out = q_out;
    a.ldk = ldk; a.ldv = ldv; a.ldq = ldq; a.ldqo = ldqo;
    a.frequencies = frequencies;
    a.tokens = (int32_t)tokens; a.heads = heads; a.pairs = pairs; a.interleaved = interleaved != 0;
    return by_type(cache->type, [&](auto type) -> int {
        using T = decltype(type);
        auto go = [&](auto width) -> int {
            constexpr int U = decltype(width)::value;
            a.by_rotated = Divider::of(pairs / U + (dim - 2 * pairs) / U);
            a.by_copied = Divider::of(dim / U);
            const unsigned workgroups = (unsigned)std::min<int64_t>(tokens, int64_t(1) << 20);
            k_paged_append<T, U><<<dim3(workgroups), kThreads, 0, (hipStream_t)stream>>>(a);
            HBP_HIP(hipGetLastError());
            return HBP_OK;
        };
        // (16 bytes a load: 10000 tokens of fp32 with eight values 75.6 us, with four 71.4; 16-bit types the other way round)
        if constexpr (sizeof(T) == 2)
            if (pairs % 8 == 0) return go(std::integral_constant<int, 8>());
        if (pairs % 4 == 0) return go(std::integral_constant<int, 4>());
        return go(std::integral_constant<int, 1>());
    });
}
