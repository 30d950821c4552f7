// Attention of new tokens over a paged cache, on the matrix cores (hbp_paged_attention).
//
// Scores are taken as S^T = K Q^T and results as O^T = V^T P^T, so that a lane of a wavefront has one query in both (lane % 16), with its softmax statistics: S^T comes out
// as four positions a lane, and with the positions of a step of 32 dealt to the instruction's rows as they are here (row r of half a is position 8 (r / 4) + 4 a + r % 4) the eight weights that a
// lane makes of them are what the second product takes from it, without a word being exchanged.  V is wanted column by column: a lane loads eight positions of D / 16 columns that lie
// together and turns them in its registers.
//
// fp32 is taken as three bf16 parts of 8 bits each, exactly, and a product as the six products of parts that matter (2^-22 of it is left out).
#pragma once

#include <algorithm>

#include "hbp_paged_attend.h"

namespace hbp {
namespace {

typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));
typedef uint16_t ushort2_t __attribute__((ext_vector_type(2)));
template <typename T, int N> using vec_t = T __attribute__((ext_vector_type(N)));

constexpr float kLowest = -3.4028234663852886e38f;
// From here on an exponent's own rounding would count: the largest one, score times `per` in fp32, is off by up to half a place (an eighth below 2^22, 64 at 2^31), and a weight that is exp2 of the exact
// product less that would be as many powers of 2 too large or too small, until the largest one overflows or vanishes.
constexpr float kFarExponent = 4194304.0f;

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }    // a's, then b's
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Eight values of a lane as an operand of the matrix instruction.
template <typename T> struct Operand {
    uint4_t w;
    static __device__ __forceinline__ Operand of(const uint32_t (&bits)[4]) { return Operand{uint4_t{bits[0], bits[1], bits[2], bits[3]}}; }
    static __device__ __forceinline__ Operand of(const float (&v)[8])   // rounded
    {
        vec_t<T, 8> r;
#pragma unroll
        for (int i = 0; i < 8; i++) r[i] = from_f32<T>(v[i]);
        return Operand{__builtin_bit_cast(uint4_t, r)};
    }
};
template <> struct Operand<float> {
    uint4_t w[3];
    static __device__ __forceinline__ Operand of(const float (&v)[8])
    {
        Operand r;
        float rest[8];
#pragma unroll
        for (int i = 0; i < 8; i++) rest[i] = v[i];
#pragma unroll
        for (int part = 0; part < 3; part++) {
#pragma unroll
            for (int i = 0; i < 4; i++) r.w[part][i] = high_halves(__float_as_uint(rest[2 * i]), __float_as_uint(rest[2 * i + 1]));
            if (part < 2)
#pragma unroll
                for (int i = 0; i < 8; i++) rest[i] -= __uint_as_float(__float_as_uint(rest[i]) & 0xffff0000u);
        }
        return r;
    }
    static __device__ __forceinline__ Operand of(const uint32_t (&bits)[8])
    {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = __uint_as_float(bits[i]);
        return of(v);
    }
};
__device__ __forceinline__ float4_t multiply_bf16(uint4_t a, uint4_t b, float4_t c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(vec_t<bf16, 8>, a), __builtin_bit_cast(vec_t<bf16, 8>, b), c, 0, 0, 0);
}
__device__ __forceinline__ float4_t multiply(const Operand<bf16> &a, const Operand<bf16> &b, float4_t c, int) { return multiply_bf16(a.w, b.w, c); }
__device__ __forceinline__ float4_t multiply(const Operand<f16> &a, const Operand<f16> &b, float4_t c, int)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(vec_t<f16, 8>, a.w), __builtin_bit_cast(vec_t<f16, 8>, b.w), c, 0, 0, 0);
}
// the products of parts that make an fp32 product, small ones first; one of them waits for the sum of the one before, so that several sums are taken in turn
template <typename T> constexpr int kProducts = sizeof(T) == 4 ? 6 : 1;
__device__ __forceinline__ float4_t multiply(const Operand<float> &a, const Operand<float> &b, float4_t c, int product)
{
    constexpr int of_a[6] = {1, 0, 2, 0, 1, 0}, of_b[6] = {1, 2, 0, 1, 0, 0};
    return multiply_bf16(a.w[of_a[product]], b.w[of_b[product]], c);
}

// a value that is the same in all lanes, as one of the wavefront's
__device__ __forceinline__ int32_t one(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint32_t one(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// over the four lanes that have the same query
template <typename F> __device__ __forceinline__ float over_quarters(float v, F op)
{
    uint32_t w = __float_as_uint(v);
    auto a = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    w = __float_as_uint(v);
    auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Exponents of 2 of scores with a cap.  tanh x = 1 - 2 / (e^2x + 1) is off by some 2^-22 of 1 also where x is small, which is as much of the cap in the exponent: fp32 results would show it, and those of 16-bit types
// with caps above kNearCap (up to there it is 3e-5 of a weight, a sixteenth of fp16's half step).
constexpr float kNearCap = 128.0f, kPerLog2 = 1.4426950408889634f;
template <typename T> __device__ __forceinline__ float capped(const Attend &a, float score)
{
    if constexpr (sizeof(T) == 4) return a.cap_out * tanhf(score * a.cap_in);
    const float e = __builtin_amdgcn_exp2f(score * (a.cap_in * (2.0f * kPerLog2)));
    return a.cap_out - 2.0f * a.cap_out * __builtin_amdgcn_rcpf(e + 1.0f);
}
template <typename T> __host__ __device__ __forceinline__ bool has_far_cap(const Attend &a) { return sizeof(T) == 2 && a.cap_out > kNearCap * kPerLog2; }
// The same of a lane's eight scores, off relative to what comes out, for 16-bit types and any cap: x below 3/8 by tanh's series, whose first term left out is 3e-8 of it there, and the others by their magnitude, 7e-7
// of it at the most.  One score after the other: it is not to cost room in the loops that it stands in.
__device__ __forceinline__ void far_capped(const Attend &a, float (&e)[8])
{
#pragma unroll 1
    for (int i = 0; i < 8; i++) {
        float score = e[0];
#pragma unroll
        for (int j = 1; j < 8; j++) score = j == i ? e[j] : score;
        const float x = score * a.cap_in, y = x * x;
        const float near = fmaf(fmaf(fmaf(fmaf(fmaf(-1382.0f / 155925.0f, y, 62.0f / 2835.0f), y, -17.0f / 315.0f), y, 2.0f / 15.0f), y, -1.0f / 3.0f), y * x, x);
        const float power = __builtin_amdgcn_exp2f(fabsf(x) * (2.0f * kPerLog2));
        const float other = copysignf(fmaf(-2.0f, __builtin_amdgcn_rcpf(power + 1.0f), 1.0f), x);
        score = a.cap_out * (fabsf(x) < 0.375f ? near : other);
#pragma unroll
        for (int j = 0; j < 8; j++) e[j] = j == i ? score : e[j];
    }
}

// A position's slot: its page (-1: not held) and the place in it
struct Slot {
    int32_t page, within;
};
__device__ __forceinline__ Slot slot_of(const Paged &c, const int32_t *table, int32_t position)
{
    const int32_t which = c.by_page.divide(position);
    const int32_t page = table[which];
    return Slot{page >= 0 && page < c.pages ? page : -1, position - which * c.page_size};
}
template <typename T> __device__ __forceinline__ const T *row_of(const void *pages, int64_t ld, const Paged &c, int32_t kv_head, Slot s)
{
    return static_cast<const T *>(pages) + (int64_t)max(s.page, 0) * ld + (int64_t)kv_head * c.page_size * c.head_dim + s.within * c.head_dim;   // (the last one is below 2^24)
}

// N values (2 to 16, 4 or more bytes) of a row in the cache: rows are 16-byte aligned
template <typename T, int N> struct Piece {
    static constexpr int kWords = N * sizeof(T) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (kWords == 1) {
            w[0] = *reinterpret_cast<const uint32_t *>(p);
        } else if constexpr (kWords == 2) {
            const uint2 v = *reinterpret_cast<const uint2 *>(p);
            w[0] = v.x; w[1] = v.y;
        } else {
#pragma unroll
            for (int i = 0; i < kWords / 4; i++) {
                const uint4 v = *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p) + 16 * i);
                w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
            }
        }
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return to_f32(__builtin_bit_cast(T, (uint16_t)(w[i / 2] >> (i & 1) * 16)));
    }
};

// Infinities and NaN among 16-bit values, two to a word, or among fp32 values
__device__ __forceinline__ uint32_t largest_halves(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2_t, a), __builtin_bit_cast(ushort2_t, b)));
}
template <typename T> constexpr uint32_t kInfinite = std::is_same_v<T, float> ? 0x7f800000u : std::is_same_v<T, f16> ? 0x7c00u : 0x7f80u;
template <typename T> __device__ __forceinline__ bool has_odd(uint32_t w)   // of words without signs
{
    return sizeof(T) == 4 ? w >= kInfinite<T> : (w & 0xffffu) >= kInfinite<T> || w >> 16 >= kInfinite<T>;
}
template <typename T> __device__ __forceinline__ uint32_t without_odd(uint32_t w)
{
    if constexpr (sizeof(T) == 4) return (w & 0x7fffffffu) >= kInfinite<T> ? 0u : w;
    const uint32_t low = (w & 0x7fffu) >= kInfinite<T> ? 0u : w & 0xffffu, high = (w >> 16 & 0x7fffu) >= kInfinite<T> ? 0u : w & 0xffff0000u;
    return low | high;
}
// Weights of a row are taken relative to an earlier largest exponent until one is kSlack above it.  In fp16 it is taken 7 less: weights are then 2^7 where they are largest, 2^15 at most, and
// small ones are rounded to multiples of 2^-24, at most 2^-31 of the largest one and not 2^-24 of it (of a long tail of weights of 2^-25.1 nothing would be left in the result, and 0.3 % in the sum).
template <typename T> constexpr float kUp = std::is_same_v<T, f16> ? 7.0f : 0.0f;
template <typename T> constexpr float kSlack = 8.0f + kUp<T>;

// Rows whose largest exponent m is far from 0 have exponents rounded as m was: their scores become those that `per` makes differences to m of, without m (less); or the weights that
// have been made of them are made again.
__device__ __forceinline__ void far_scores(float (&e)[8], float m, float per, float &less)
{
    if (!(fabsf(m) >= kFarExponent)) return;
    less = 0.0f;
    const float inverse = 1.0f / per;
#pragma unroll
    for (int i = 0; i < 8; i++) {
#pragma clang fp contract(off)
        const float exponent = e[i] * per;
        e[i] = (exponent - m) * inverse;
    }
}
__device__ __forceinline__ void far_weights(float (&p)[8], const float (&e)[8], float m, float per)
{
    const bool far = fabsf(m) >= kFarExponent;
#pragma unroll
    for (int i = 0; i < 8; i++) {
#pragma clang fp contract(off)
        const float exponent = e[i] * per;
        p[i] = far ? __builtin_amdgcn_exp2f(exponent - m) : p[i];
    }
}

// The weight of position t of a step for the lane's query, from the lane that has it
template <typename T> __device__ __forceinline__ float weight_of(const Operand<T> &weights, int t, int column)
{
    uint32_t w[3];
#pragma unroll
    for (int part = 0; part < (sizeof(T) == 4 ? 3 : 1); part++) {
        const uint4_t *from = reinterpret_cast<const uint4_t *>(&weights) + part;
        const uint32_t mine = t / 2 % 4 == 0 ? (*from)[0] : t / 2 % 4 == 1 ? (*from)[1] : t / 2 % 4 == 2 ? (*from)[2] : (*from)[3];
        w[part] = (uint32_t)__shfl((int)mine, t / 8 * 16 + column) >> (t & 1) * 16 & 0xffffu;
    }
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[0] << 16) + __uint_as_float(w[1] << 16) + __uint_as_float(w[2] << 16);
    else return to_f32(__builtin_bit_cast(T, (uint16_t)w[0]));
}

// fp32: parts of an infinite value, and products of parts that overflow, make NaN of what may be a number or an infinity.  Scores of a lane's eight positions of a step that are not finite are computed
// again where its query sees them (`held`: bits of those that the cache holds).
__device__ __forceinline__ void by_definition(const Attend &a, const Unit &x, const int32_t *table, int32_t kv_head, int32_t row, int32_t step, int32_t low, int32_t count, uint32_t held, float (&e)[8])
{
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) odd |= !(fabsf(e[i]) < INFINITY) ? 1u << i : 0u;
    if (__ballot(odd != 0) == 0) return;
    const int32_t first = step + 8 * ((int)threadIdx.x % kWave / 16);
    odd &= held;
    if (odd == 0 || count <= 0) return;
    const int32_t token = a.by_group.divide(row);
    const float *query = static_cast<const float *>(a.q) + (int64_t)(x.first_token + token) * a.ldq + (int64_t)(kv_head * a.group + row - token * a.group) * a.c.head_dim;
#pragma unroll 1
    for (int i = 0; i < 8; i++) {
        if (!(odd >> i & 1) || (uint32_t)(first + i - low) >= (uint32_t)count) continue;
        const float *key = row_of<float>(a.c.keys, a.c.ldk, a.c, kv_head, slot_of(a.c, table, first + i));
        float sum = 0.0f;
#pragma unroll 1
        for (int d = 0; d < a.c.head_dim && sum == sum; d++) sum += query[d] * key[d];
        sum = a.flip ? -sum : sum;
#pragma unroll
        for (int j = 0; j < 8; j++) e[j] = j == i ? sum : e[j];
    }
}

// Adds the infinities and NaN among the values of positions from..to - 1 of a step, for the queries that see them.  (Hardly ever called: it is not to cost registers elsewhere.)
template <typename T, int D, int NQ>
__device__ __forceinline__ void add_odd(const Attend &a, const int32_t *table, int32_t kv_head, int32_t step, int32_t from, int32_t to, const Operand<T> (&weights)[NQ],
                                        const int32_t (&low)[NQ], const int32_t (&count)[NQ], float4_t (&o)[NQ][D / 16])
{
    constexpr int kTiles = D / 16, kEach = kTiles > 8 ? 8 : kTiles;
    const int lane = threadIdx.x % kWave, column = lane % 16;
#pragma unroll 1
    for (int32_t position = from; position < to; position++) {
        const Slot slot = slot_of(a.c, table, position);
        if (slot.page < 0) continue;
        const T *values = row_of<T>(a.c.values, a.c.ldv, a.c, kv_head, slot);
        float weight[NQ];   // (of all lanes, before some of them leave: a lane that is switched off has nothing to give)
#pragma unroll
        for (int n = 0; n < NQ; n++) weight[n] = weight_of(weights[n], position - step, column);
        int32_t at = kTiles * 4 * (lane / 16);
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
            for (int c = 0; c < kTiles; c += kEach) {
                asm volatile("" : "+v"(at) : : "memory");   // (one load after the other, nothing worked out before the loop)
                Piece<T, kEach> v;
                const int32_t d = at + kTiles * k + c;
                if (d >= a.c.head_dim) continue;
                v.load(values + d);
#pragma unroll
                for (int n = 0; n < NQ; n++) {
                    const bool sees = (uint32_t)(position - low[n]) < (uint32_t)count[n];
#pragma unroll
                    for (int i = 0; i < kEach; i++) {
                        const float value = v.get(i);
                        if (sees && !(fabsf(value) < INFINITY)) o[n][c + i][k] += weight[n] * value;
                    }
                }
            }
    }
}

// Few rows: a workgroup of four wavefronts takes 16 NQ rows, and each wavefront every fourth step of their positions, straight from the cache into registers; the four
// results are joined in LDS.  The next step's keys are on their way from the scores on, this one's values until the weights are there.  Bound: HBM where there are many positions (64 sequences over up
// to 16000, fp16, heads of 128: 396 us, 5.8 TB/s), its latency with heads of 256, whose 32 KB of a step leave two wavefronts a SIMD (24 x 5 tokens, a window of 4096: 152 us, 5.3 TB/s), and a chain of
// loads (starts, the table, keys) with few: 6.7 us for one token over 4096.  Nothing is shared in LDS: with at most 32 rows no wavefront would read what another one has loaded.
template <typename T, int D, int NQ, bool ANY_PAGE> __global__ __launch_bounds__(256, sizeof(T) == 4 && D > 64 ? 1 : 2) void k_attend(Attend a, int64_t first_unit)
{
    constexpr int kSteps = D / 32, kTiles = D / 16;   // of 32 columns in Q K^T; of 16 in the result, which a lane holds D / 16 neighbouring columns of
    constexpr int kPitch = D + 4, kSums = sizeof(T) == 4 && D < 256 ? 2 : 1;   // sums taken in turn
    constexpr bool kAhead = D <= 128;   // whether the next step's keys are on their way beside this one's values: with wider heads they would take the registers of a second wavefront (16 bits: 171 and 166 us for 24 x 5 x 4096)
    __shared__ float joined[4][16][kPitch];
    __shared__ float2 joined_stats[4][16];
    const int lane = threadIdx.x % kWave, wave = one((int32_t)threadIdx.x / kWave), column = lane % 16, quarter = lane / 16;
    const int64_t number = first_unit + blockIdx.x;
    const int32_t unit_number = (int32_t)(number / a.c.kv_heads), kv_head = (int32_t)(number - (int64_t)unit_number * a.c.kv_heads);
    Unit x;
    if (!find_unit<false, 256>(a, unit_number, x)) return;
    const int32_t begin = x.low + x.part * x.size, end = min(begin + x.size, x.high);
    const int32_t *table = a.c.table + x.sequence * a.c.ldt;
    const int32_t dim = a.c.head_dim;

    Operand<T> q[NQ][kSteps];
    int32_t low[NQ], count[NQ];   // the positions that the lane's query sees: low .. low + count - 1
    int32_t all_low = 0, all_high = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < NQ; n++) {
        const int32_t row = x.tile * a.tile_rows + n * 16 + column;
        const bool is_row = row < x.rows;
        const int32_t token = a.by_group.divide(is_row ? row : 0), head = kv_head * a.group + (is_row ? row - token * a.group : 0);
        const T *from = static_cast<const T *>(a.q) + (int64_t)(x.first_token + token) * a.ldq + (int64_t)head * dim;
#pragma unroll
        for (int k = 0; k < kSteps; k++) {
            const int32_t at = 32 * k + 8 * quarter;
            Eight<T> v;
            v.clear();
            if (is_row && at < dim) v.load(from + at);
#pragma unroll
            for (int i = 0; i < Eight<T>::kWords; i++) v.w[i] = (v.w[i] & a.keep) ^ a.flip;
            q[n][k] = Operand<T>::of(v.w);
        }
        const int64_t position = x.first_position + token;
        low[n] = (int32_t)max((int64_t)0, a.window ? position - a.window + 1 : 0);
        const int32_t high = (int32_t)max((int64_t)0, min(position + 1, (int64_t)end));
        count[n] = is_row ? max(0, high - low[n]) : 0;
        if (is_row) {
            all_low = max(all_low, low[n]);
            all_high = min(all_high, high);
        }
    }
    all_low = one(wave_reduce(all_low, [](int32_t p, int32_t q) { return max(p, q); }));
    all_high = one(wave_reduce(all_high, [](int32_t p, int32_t q) { return min(p, q); }));
    const int32_t least_low = x.low;   // (a multiple of kStep: positions from there to the window's are seen by no row, and their values have to go)
    int32_t tile_low = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < NQ; n++) tile_low = min(tile_low, count[n] ? low[n] : 0x7fffffff);
    tile_low = max(least_low, one(wave_reduce(tile_low, [](int32_t p, int32_t q) { return min(p, q); })));

    const float per = a.cap_out != 0.0f ? 1.0f : a.per;   // (of what the cap has made of scores)
    float m[NQ], l[NQ];
    float4_t o[NQ][kTiles];
    int32_t far[NQ];   // whether a row's largest exponent is far from 0 (the same in all lanes)
#pragma unroll
    for (int n = 0; n < NQ; n++) {
        m[n] = kLowest;
        l[n] = 0.0f;
        far[n] = 0;
#pragma unroll
        for (int j = 0; j < kTiles; j++) o[n][j] = float4_t{0, 0, 0, 0};
    }

    // what a lane loads of a step: as rows of K, positions 8 (column / 4) + column % 4 and 4 more; as columns of V, 8 quarter + 0..7
    struct Places {
        Slot k[ANY_PAGE ? 2 : 1], v[ANY_PAGE ? 8 : 1];
    };
    auto places = [&](int32_t step) {   // (of positions moved back before the end: what is read there has no weight)
        Places r;
        if constexpr (ANY_PAGE) {
#pragma unroll
            for (int h = 0; h < 2; h++) r.k[h] = slot_of(a.c, table, min(step + 8 * (column / 4) + 4 * h + column % 4, end - 1));
#pragma unroll
            for (int i = 0; i < 8; i++) r.v[i] = slot_of(a.c, table, min(step + 8 * quarter + i, end - 1));
        } else {
            const int32_t last = (end - 1) / 8 * 8;   // (eight positions from a multiple of 8 on are in one page)
            r.k[0] = slot_of(a.c, table, min(step + 8 * (column / 4), last));
            r.v[0] = slot_of(a.c, table, min(step + 8 * quarter, last));
        }
        return r;
    };
    Piece<T, 8> kf[2][kSteps];
    auto load_keys = [&](const Places &p) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const T *from = ANY_PAGE ? row_of<T>(a.c.keys, a.c.ldk, a.c, kv_head, p.k[ANY_PAGE ? h : 0])
                                     : row_of<T>(a.c.keys, a.c.ldk, a.c, kv_head, p.k[0]) + (4 * h + column % 4) * dim;
#pragma unroll
            for (int k = 0; k < kSteps; k++) {
                const int32_t at = 32 * k + 8 * quarter;
                kf[h][k].load(from + (at < dim ? at : 0));
            }
        }
    };

    if (begin < end) {
        int32_t step = begin + wave * kStep;
        Places now = places(step), next = places(step + 4 * kStep);
        if constexpr (kAhead) load_keys(now);
        for (; step < end; step += 4 * kStep) {
            constexpr int kPieces = kTiles > 8 ? kTiles / 8 : 1, kEach = kTiles > 8 ? 8 : kTiles;
            Piece<T, kEach> vf[8][kPieces];
            auto load_values = [&](const Places &p) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const T *from = ANY_PAGE ? row_of<T>(a.c.values, a.c.ldv, a.c, kv_head, p.v[ANY_PAGE ? i : 0])
                                             : row_of<T>(a.c.values, a.c.ldv, a.c, kv_head, p.v[0]) + i * dim;
#pragma unroll
                    for (int c = 0; c < kPieces; c++) {
                        const int32_t at = kTiles * column + kEach * c;
                        vf[i][c].load(from + (at < dim ? at : 0));
                    }
                }
            };
            if constexpr (kAhead) load_values(now);
            else load_keys(now);
            // scores
            float4_t s[NQ][2];
#pragma unroll
            for (int n = 0; n < NQ; n++) s[n][0] = s[n][1] = float4_t{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < kSteps; k++) {
                const uint32_t there = 32 * k + 8 * quarter < dim ? 0xffffffffu : 0u;
                Operand<T> key[2];
#pragma unroll
                for (int h = 0; h < 2; h++) {
#pragma unroll
                    for (int i = 0; i < Piece<T, 8>::kWords; i++) kf[h][k].w[i] &= there;
                    key[h] = Operand<T>::of(kf[h][k].w);
                }
#pragma unroll
                for (int product = 0; product < kProducts<T>; product++)
#pragma unroll
                    for (int h = 0; h < 2; h++)
#pragma unroll
                        for (int n = 0; n < NQ; n++) s[n][h] = multiply(key[h], q[n][k], s[n][h], product);
            }
            const Places mine = now;
            now = next;
            if constexpr (kAhead) load_keys(now);
            else load_values(mine);
            next = places(step + 8 * kStep);

            uint32_t held = 0;   // bits of the lane's eight positions that the cache holds
#pragma unroll
            for (int i = 0; i < 8; i++) held |= mine.v[ANY_PAGE ? i : 0].page >= 0 ? 1u << i : 0u;
            const bool whole = step >= all_low && step + kStep <= all_high && __ballot(held != 0xff) == 0;   // every row sees every position

            Operand<T> weights[NQ];
#pragma unroll
            for (int n = 0; n < NQ; n++) {
                float e[8], p[8];
#pragma unroll
                for (int i = 0; i < 8; i++) e[i] = s[n][i / 4][i % 4];
                if constexpr (sizeof(T) == 4) by_definition(a, x, table, kv_head, x.tile * a.tile_rows + n * 16 + column, step, low[n], count[n], held, e);
                if (a.cap_out != 0.0f) {
                    if (has_far_cap<T>(a))
                        far_capped(a, e);
                    else
#pragma unroll
                        for (int i = 0; i < 8; i++) e[i] = capped<T>(a, e[i]);
                }
                if (!whole)
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const bool sees = (uint32_t)(step + 8 * quarter + i - low[n]) < (uint32_t)count[n] && (held >> i & 1);
                        e[i] = sees ? e[i] : -INFINITY;
                    }
                float top = e[0];
#pragma unroll
                for (int i = 1; i < 8; i++) top = fmaxf(top, e[i]);
                top *= per;
                // The weights are taken relative to an earlier largest exponent while none is more than kSlack above it (by the difference, which is exact): sums stay far from overflow, and nothing is exchanged.
                if (__ballot(top - m[n] > kSlack<T>) != 0) {
                    const float to = over_quarters(fmaxf(top - kUp<T>, m[n]), [](float p, float q) { return fmaxf(p, q); });
                    const float f = __builtin_amdgcn_exp2f(m[n] - to);
                    m[n] = to;
                    far[n] = __ballot(fabsf(to) >= kFarExponent && to > kLowest) != 0;
                    l[n] *= f;
#pragma unroll
                    for (int j = 0; j < kTiles; j++)
#pragma unroll
                        for (int i = 0; i < 4; i++) o[n][j][i] *= f;
                }
#pragma unroll
                for (int i = 0; i < 8; i++) p[i] = __builtin_amdgcn_exp2f(fmaf(e[i], per, -m[n]));   // (the exponent is rounded as a difference to the largest one)
                if (one(far[n])) far_weights(p, e, m[n], per);
#pragma unroll
                for (int i = 0; i < 8; i++) l[n] += p[i];
                weights[n] = Operand<T>::of(p);
            }

            // Values that no row sees must not be there at all, not even with a weight of 0; infinities and NaN are taken out where only some rows see them (in fp32 everywhere:
            // parts of an infinity make NaN), and added for those rows.
            bool odd = false;
            if (!whole || sizeof(T) == 4) {
                uint32_t largest = 0;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const int32_t position = step + 8 * quarter + i;
                    const uint32_t seen = position >= tile_low && position < end && (held >> i & 1) ? 0xffffffffu : 0u;
#pragma unroll
                    for (int c = 0; c < kPieces; c++)
#pragma unroll
                        for (int w = 0; w < Piece<T, kEach>::kWords; w++) {
                            vf[i][c].w[w] &= seen;
                            if constexpr (sizeof(T) == 4) largest = max(largest, vf[i][c].w[w] & 0x7fffffffu);
                            else largest = largest_halves(largest, vf[i][c].w[w] & 0x7fff7fffu);
                        }
                }
                odd = __ballot(has_odd<T>(largest)) != 0;
                if (odd)
#pragma unroll
                    for (int i = 0; i < 8; i++)
#pragma unroll
                        for (int c = 0; c < kPieces; c++)
#pragma unroll
                            for (int w = 0; w < Piece<T, kEach>::kWords; w++) vf[i][c].w[w] = without_odd<T>(vf[i][c].w[w]);
            }
#pragma unroll
            for (int j = 0; j < kTiles; j += kSums) {
                Operand<T> value[kSums];
#pragma unroll
                for (int c = 0; c < kSums; c++) {
                    const int at = j + c;
                    if constexpr (sizeof(T) == 4) {
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; i++) v[i] = __uint_as_float(vf[i][at / kEach].w[at % kEach]);
                        value[c] = Operand<T>::of(v);
                    } else {
                        uint32_t bits[4];
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            const uint32_t one = vf[2 * i][at / kEach].w[at % kEach / 2], two = vf[2 * i + 1][at / kEach].w[at % kEach / 2];
                            bits[i] = at & 1 ? high_halves(one, two) : low_halves(one, two);
                        }
                        value[c] = Operand<T>::of(bits);
                    }
                }
#pragma unroll
                for (int product = 0; product < kProducts<T>; product++)
#pragma unroll
                    for (int c = 0; c < kSums; c++)
#pragma unroll
                        for (int n = 0; n < NQ; n++) o[n][j + c] = multiply(value[c], weights[n], o[n][j + c], product);
            }
            if (odd) {
                add_odd<T, D, NQ>(a, table, kv_head, step, max(tile_low, step), min(end, step + kStep), weights, low, count, o);
            }
        }
    }

    // the four wavefronts' sums
#pragma unroll
    for (int n = 0; n < NQ; n++) {
        l[n] = over_quarters(l[n], [](float p, float q) { return p + q; });
        if (n) __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
            for (int j = 0; j < kTiles; j++) joined[wave][column][kTiles * (4 * quarter + k) + j] = o[n][j][k];
        if (quarter == 0) joined_stats[wave][column] = float2{m[n], l[n]};
        __syncthreads();
        constexpr int kChunks = D / 8;
        for (int i = threadIdx.x; i < 16 * kChunks; i += 256) {
            const int r = i / kChunks, at = i % kChunks * 8;
            const int32_t row = x.tile * a.tile_rows + n * 16 + r;
            if (row >= x.rows || at >= dim) continue;
            float top = kLowest, sum = 0.0f, v[8] = {};
#pragma unroll
            for (int w = 0; w < 4; w++) top = fmaxf(top, joined_stats[w][r].x);
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float2 stats = joined_stats[w][r];
                const float f = __builtin_amdgcn_exp2f(stats.x - top);
                sum += stats.y * f;
#pragma unroll
                for (int k = 0; k < 8; k++) v[k] += joined[w][r][at + k] * f;
            }
            if (x.parts == 1) {
                const int32_t token = a.by_group.divide(row);
                Eight<T> out;
                const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
                for (int k = 0; k < 8; k++) out.set(k, sum == 0.0f ? 0.0f : v[k] * inverse);
                out.store(static_cast<T *>(a.out) + (int64_t)(x.first_token + token) * a.ldo + (int64_t)(kv_head * a.group + row - token * a.group) * dim + at);
            } else {
                const int64_t to = ((int64_t)(x.slot + x.part) * a.c.kv_heads + kv_head) * a.tile_rows + n * 16 + r;
                float4 *sums = reinterpret_cast<float4 *>(a.partial + to * dim + at);
                sums[0] = float4{v[0], v[1], v[2], v[3]};
                sums[1] = float4{v[4], v[5], v[6], v[7]};
                if (at == 0) a.partial_stats[to] = float2{top, sum};
            }
        }
    }
}

// Joins the parts of tiles that were split: a workgroup sixteen rows of a tile, LANES lanes a part of a row with eight columns each.  A wavefront has ROWS rows at once, or one with as many parts
// on their way: what it waits for is the latency of loads: 4.9 us for one token over 4096 positions, 15 for 512 of 32 heads over
// 30000.  The grid is as large as the lengths could make it: 28 us for the 13696 workgroups behind 4 x 2048 tokens over up to 8000, whose 832 tiles are all whole, so that none of them has anything to join.
template <typename T, int LANES, int ROWS> __global__ __launch_bounds__(256) void k_attend_join(Attend a, int64_t first)
{
    constexpr int kAtOnce = kWave / LANES, kAhead = 4 / ROWS;   // parts side by side, and one behind the other on their way
    const int64_t number = first + blockIdx.x;
    const int32_t groups = a.tile_rows / 16, dim = a.c.head_dim;
    const int64_t tile_head = number / groups;
    const int32_t n = (int32_t)(number - tile_head * groups), tile = (int32_t)(tile_head / a.c.kv_heads), kv_head = (int32_t)(tile_head - (int64_t)tile * a.c.kv_heads);
    Unit x;
    if (!find_unit<true, 256>(a, tile, x) || x.parts == 1) return;
    const int32_t span = max(0, x.high - x.low), parts = x.size ? (span + x.size - 1) / x.size : 0;   // (those with positions)
    const int lane = threadIdx.x % kWave, wave = one((int32_t)threadIdx.x / kWave), which = lane / LANES, at = lane % LANES * 8;
    const bool mine = at < dim;
    const int64_t apart = (int64_t)a.c.kv_heads * a.tile_rows;
    const int32_t tile_row = n * 16, left = x.rows - x.tile * a.tile_rows - tile_row;   // (rows from there on that the sequence has)
    for (int r0 = wave; r0 < min(16, left); r0 += 4 * ROWS) {
        float top[ROWS], sum[ROWS], v[ROWS][8];
        int64_t from[ROWS];
#pragma unroll
        for (int q = 0; q < ROWS; q++) {
            from[q] = ((int64_t)x.slot * a.c.kv_heads + kv_head) * a.tile_rows + tile_row + min(r0 + 4 * q, left - 1);   // (rows that are not there are read as the last one, for nothing)
            top[q] = kLowest;
            sum[q] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; i++) v[q][i] = 0.0f;
        }
        for (int32_t p0 = which; p0 < parts; p0 += kAtOnce * kAhead) {
            float2 stats[ROWS][kAhead];
            float4 part[ROWS][kAhead][2];
#pragma unroll
            for (int q = 0; q < ROWS; q++)
#pragma unroll
                for (int k = 0; k < kAhead; k++) {
                    const int32_t p = p0 + k * kAtOnce;
                    stats[q][k] = float2{kLowest, 0.0f};
                    part[q][k][0] = part[q][k][1] = float4{0, 0, 0, 0};
                    if (p < parts) {
                        stats[q][k] = a.partial_stats[from[q] + p * apart];
                        const float4 *sums = reinterpret_cast<const float4 *>(a.partial + (from[q] + p * apart) * dim + (mine ? at : 0));
                        part[q][k][0] = sums[0];
                        part[q][k][1] = sums[1];
                    }
                }
#pragma unroll
            for (int q = 0; q < ROWS; q++) {
                float higher = top[q];
#pragma unroll
                for (int k = 0; k < kAhead; k++) higher = fmaxf(higher, stats[q][k].x);
                const float f = __builtin_amdgcn_exp2f(top[q] - higher);
                top[q] = higher;
                sum[q] *= f;
#pragma unroll
                for (int i = 0; i < 8; i++) v[q][i] *= f;
#pragma unroll
                for (int k = 0; k < kAhead; k++) {
                    const float g = __builtin_amdgcn_exp2f(stats[q][k].x - higher);
                    sum[q] += stats[q][k].y * g;
                    const float4 one = part[q][k][0], two = part[q][k][1];
                    v[q][0] += one.x * g; v[q][1] += one.y * g; v[q][2] += one.z * g; v[q][3] += one.w * g;
                    v[q][4] += two.x * g; v[q][5] += two.y * g; v[q][6] += two.z * g; v[q][7] += two.w * g;
                }
            }
        }
#pragma unroll
        for (int q = 0; q < ROWS; q++) {
            float higher = top[q];
#pragma unroll
            for (int d = LANES; d < kWave; d *= 2) higher = fmaxf(higher, __shfl_xor(higher, d));
            const float f = __builtin_amdgcn_exp2f(top[q] - higher);
            sum[q] *= f;
#pragma unroll
            for (int i = 0; i < 8; i++) v[q][i] *= f;
#pragma unroll
            for (int d = LANES; d < kWave; d *= 2) {
                sum[q] += __shfl_xor(sum[q], d);
#pragma unroll
                for (int i = 0; i < 8; i++) v[q][i] += __shfl_xor(v[q][i], d);
            }
            const int r = r0 + 4 * q;
            if (which || !mine || r >= min(16, left)) continue;
            const int32_t row = x.tile * a.tile_rows + tile_row + r, token = a.by_group.divide(row);
            Eight<T> out;
            const float inverse = 1.0f / sum[q];
#pragma unroll
            for (int k = 0; k < 8; k++) out.set(k, sum[q] == 0.0f ? 0.0f : v[q][k] * inverse);
            out.store(static_cast<T *>(a.out) + (int64_t)(x.first_token + token) * a.ldo + (int64_t)(kv_head * a.group + row - token * a.group) * dim + at);
        }
    }
}

template <typename T, int D, int NQ, bool ANY_PAGE> int launch_units(const Attend &a, hipStream_t st)
{
    constexpr int64_t kMost = int64_t(1) << 23;   // workgroups of one launch: a grid's threads are counted in 32 bits
    const int64_t units = a.units * a.c.kv_heads;
    for (int64_t at = 0; at < units; at += kMost) {
        k_attend<T, D, NQ, ANY_PAGE><<<dim3((unsigned)std::min(units - at, kMost)), 256, 0, st>>>(a, at);
        HBP_HIP(hipGetLastError());
    }
    return HBP_OK;
}

}  // namespace
}  // namespace hbp
