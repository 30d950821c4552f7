// Products y = x W^T with a matrix in 4 bits, on the matrix cores (hbp_q4_mv).
//
// With x of 16 bits a code q becomes the number 16 + q by putting its four bits at the top of the mantissa of 16, in bf16 or fp16, exactly: one shift and one
// and-or for two codes.  The matrix instruction multiplies them with x and sums in fp32; the 16, and the zero point, are taken out
// of a group's sum as (16 + zero) times the group's sum of x, which the same instruction gives with a constant for the codes.  Then the group's sum is
// multiplied by its scale, in fp32: no weight is ever rounded.  On the way stand sums as large as 24 sum x of a group: off, for an x all of one sign, by some 1e-5 of a result,
// which is a hundredth of what 16 bits of x and of the result are off by.
//
// With an fp32 x that would show, and a code becomes q itself as a bf16: as a byte of an fp8 number of four bits of exponent, whose values up to 15 steps of the smallest one lie evenly, it
// is q steps, and one conversion makes two codes of two of them.  Behind each 32 columns the zero point is taken off with a second instruction, of x with -zero as a bf16, so that
// nothing larger than those columns' own sum of zero x stands on the way.  What of a zero point eight bits do not hold, if anything, is taken out of a group's sum as above.
//
// The instruction's 16 rows on the side of x are "slots".  A vector of fp16 or bf16 takes one; one of fp32 is split into three bf16 parts
// of 8 bits of the mantissa each, exactly, and takes three, whose sums are added at the end.  The 16 columns on the side of the weights are
// 16 rows of the matrix.
//
// What is larger on the way than in the end: (16 + q) x or (q - zero) x, before the scale.  Where that, or a value of x itself, is infinite
// or NaN, the result is not finite, and such a result is computed again from the definition, (scale (q - zero)) x.
#pragma once

#include <algorithm>

#include "hbp_q4.h"

namespace hbp {
namespace {

typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef bf16 bf16x2_t __attribute__((ext_vector_type(2)));

template <typename MT> struct Cores;
template <> struct Cores<bf16> {
    typedef bf16 vec __attribute__((ext_vector_type(8)));
    static constexpr uint32_t kSixteen = 0x41804180u, kMask = 0x00780078u, kOne = 0x3f803f80u, kMinus24 = 0xc1c0c1c0u;
    static constexpr int kUp = 3;  // the lowest bit of the four top bits of the mantissa
    static __device__ __forceinline__ float4_t mul(uint4_t a, uint4_t b, float4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(vec, a), __builtin_bit_cast(vec, b), c, 0, 0, 0);
    }
};
template <> struct Cores<f16> {
    typedef f16 vec __attribute__((ext_vector_type(8)));
    static constexpr uint32_t kSixteen = 0x4c004c00u, kMask = 0x03c003c0u, kOne = 0x3c003c00u, kMinus24 = 0xce00ce00u;
    static constexpr int kUp = 6;
    static __device__ __forceinline__ float4_t mul(uint4_t a, uint4_t b, float4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(vec, a), __builtin_bit_cast(vec, b), c, 0, 0, 0);
    }
};

// Eight codes of a word as 16 + q, in the order 0 4 1 5 2 6 3 7 (x is staged in the same order).  The constants come in registers, which makes and-or one instruction.
struct Constants {
    uint32_t mask, sixteen;
    template <typename C> static __device__ __forceinline__ Constants of()
    {
        Constants c{C::kMask, C::kSixteen};
        asm("" : "+s"(c.mask));
        asm("" : "+v"(c.sixteen));
        return c;
    }
};
template <typename MT> __device__ __forceinline__ uint4_t numbers_of(uint32_t w, Constants k)
{
    using C = Cores<MT>;
    uint4_t r;
    r.x = (w << C::kUp & k.mask) | k.sixteen;
    r.y = ((C::kUp >= 4 ? w << (C::kUp - 4) : w >> (4 - C::kUp)) & k.mask) | k.sixteen;
    r.z = (w >> (8 - C::kUp) & k.mask) | k.sixteen;
    r.w = (w >> (12 - C::kUp) & k.mask) | k.sixteen;
    return r;
}

// Eight codes of a word as they are, in bf16, in the order 0 2 4 6 1 3 5 7 (which an fp32 x is staged in).  512: the steps of an fp8 number of four bits of exponent are 1 / 512.
__device__ __forceinline__ uint4_t codes_of(uint32_t w)
{
    const uint32_t even = w & 0x0f0f0f0fu, odd = w >> 4 & 0x0f0f0f0fu;
    uint4_t r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, 512.0f, false));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, 512.0f, true));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, 512.0f, false));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, 512.0f, true));
    return r;
}

// Four words of each lane, exchanged between the four quarters of a wavefront: word j of quarter q becomes word q of quarter j.
__device__ __forceinline__ void transpose_quarters(uint4_t &w)
{
    auto a = __builtin_amdgcn_permlane32_swap(w.x, w.z, false, false);
    auto b = __builtin_amdgcn_permlane32_swap(w.y, w.w, false, false);
    auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    w.x = c[0]; w.y = c[1]; w.z = d[0]; w.w = d[1];
}

// One output from the definition, by a wavefront: where the way over 16 + q is not finite.
template <typename T, typename S> __device__ __forceinline__ float by_definition(const Q4Product &p, int64_t row, int64_t vector)
{
    const uint8_t *codes = p.a.codes + row * p.a.pitch;
    const S *scales = static_cast<const S *>(p.a.scales) + row * p.a.groups, *zeros = static_cast<const S *>(p.a.zeros) + row * p.a.groups;
    float sum = 0;
    for (int k = threadIdx.x % kWave; k < p.a.n_cols; k += kWave) {
        const float q = (float)(codes[k / 2] >> (k & 1) * 4 & 15);
        const float zero = p.a.zeros ? to_f32(zeros[k >> p.a.shift]) : 8.0f;
        sum += to_f32(scales[k >> p.a.shift]) * (q - zero) * to_f32(static_cast<const T *>(p.x)[vector * p.ldx + k]);
    }
    return wave_sum(sum);
}

// Eight values of x on their way into LDS: as one part in the order of numbers_of, or as three in that of codes_of.
template <typename T> struct Staged {
    Eight<T> v;
    __device__ __forceinline__ void store(uint32_t *at, int words_to_next_part)
    {
        uint4_t w;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int part = 0; part < 3; part++) {
                w.x = (v.w[0] >> 16) | (v.w[2] & 0xffff0000u);
                w.y = (v.w[4] >> 16) | (v.w[6] & 0xffff0000u);
                w.z = (v.w[1] >> 16) | (v.w[3] & 0xffff0000u);
                w.w = (v.w[5] >> 16) | (v.w[7] & 0xffff0000u);
                *reinterpret_cast<uint4_t *>(at + part * words_to_next_part) = w;
#pragma unroll
                for (int i = 0; i < 8; i++) v.w[i] = __float_as_uint(__uint_as_float(v.w[i]) - __uint_as_float(v.w[i] & 0xffff0000u));
            }
        } else {
            w.x = (v.w[0] & 0xffffu) | v.w[2] << 16;
            w.y = (v.w[0] >> 16) | (v.w[2] & 0xffff0000u);
            w.z = (v.w[1] & 0xffffu) | v.w[3] << 16;
            w.w = (v.w[1] >> 16) | (v.w[3] & 0xffff0000u);
            *reinterpret_cast<uint4_t *>(at) = w;
        }
    }
};

// Loads are issued without conditions, from addresses moved back into the arrays where need be: a load that only some paths issue would
// make the compiler wait for more than it has to behind it.  Whatever is read in place of what is not there meets an x of 0.  Addresses are
// one for the wavefront, in scalar registers, and 32 bits a lane.

// N values (1, 2, 4, 8 or 16) in as few loads as can be, whatever their alignment.
typedef uint32_t one_at_2 __attribute__((aligned(2)));
typedef uint32_t two_at_2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t two_at_4 __attribute__((ext_vector_type(2), aligned(4)));
template <typename S, int N> __device__ __forceinline__ void load_values(S (&v)[N], const char *at)
{
    constexpr int kBytes = N * (int)sizeof(S);
    if constexpr (kBytes >= 16) {
        using four = std::conditional_t<sizeof(S) == 2, words_at_2, words_at_4>;
#pragma unroll
        for (int i = 0; i < kBytes / 16; i++) {
            const four w = reinterpret_cast<const four *>(at)[i];
            __builtin_memcpy(&v[i * (16 / sizeof(S))], &w, 16);
        }
    } else if constexpr (kBytes == 8) {
        using two = std::conditional_t<sizeof(S) == 2, two_at_2, two_at_4>;
        const two w = *reinterpret_cast<const two *>(at);
        __builtin_memcpy(v, &w, 8);
    } else if constexpr (kBytes == 4 && sizeof(S) == 2) {
        const uint32_t w = *reinterpret_cast<const one_at_2 *>(at);
        __builtin_memcpy(v, &w, 4);
    } else {
        static_assert(N == 1, "");
        v[0] = *reinterpret_cast<const S *>(at);
    }
}

// The scales (or zero points) of a lane's row that a batch needs: N of them, kept as they are stored until they are used.  (One load for a
// batch of several chunks: sixteen rows are sixteen lines of the cache, whatever is taken of each.)
template <typename S, int N> struct Scales {
    S v[N];
    // first: of the row's groups; inside: N values from there on are in the array for every row of the tile (what lies beyond the row's own is finite
    // or, if not, makes the result one that is computed again)
    __device__ __forceinline__ void load(const void *all, int64_t tile_at, uint32_t lane_at, int first, int groups, bool inside)
    {
        const char *at = static_cast<const char *>(all) + tile_at * (int64_t)sizeof(S);
        if (inside) {
            load_values(v, at + first * sizeof(S) + lane_at);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++) v[i] = *reinterpret_cast<const S *>(at + min(first + i, groups - 1) * sizeof(S) + lane_at);
        }
    }
};

// Where a lane finds its row of a tile of 16: bytes from the tile's first row on.  A lane takes 16 bytes of a chunk's 64, by its quarter of the wavefront.
template <typename S> struct Place {
    uint32_t codes, codes_last, scales;  // codes_last: in the last chunk, whose later quarters need not be there
    int64_t row;                         // the tile's first row, one for the wavefront
    __device__ __forceinline__ void at(const Q4 &a, int64_t first_row)
    {
        const int lane = threadIdx.x % kWave, quarter = lane >> 4;
        row = min(first_row, (int64_t)a.n_rows - 1);
        const uint32_t r = (uint32_t)min((int64_t)(lane & 15), a.n_rows - 1 - row);
        const int last_quarter = (int)(a.pitch / 16 - 1) & 3;
        codes = r * (uint32_t)a.pitch + quarter * 16;
        codes_last = r * (uint32_t)a.pitch + min(quarter, last_quarter) * 16;
        scales = r * (uint32_t)(a.groups * sizeof(S));
    }
};

// What a wavefront loads for U chunks of RT tiles.
template <typename S, bool ZERO, int GM, int RT, int U> struct Batch {
    static constexpr int N = 4 / GM;
    uint4_t words[U][RT];
    Scales<S, N * U> scale[RT], zero[ZERO ? RT : 1];
    // (chunk0 is a multiple of U, and U * 128 columns are of one group or of whole ones)
    __device__ __forceinline__ void load(const Q4 &a, const Place<S> (&place)[RT], int chunk0)
    {
        const int last = (a.n_cols + 127) / 128 - 1, first = min(chunk0, last) * 128 >> a.shift;
#pragma unroll
        for (int t = 0; t < RT; t++) {
            const bool inside = min(place[t].row + 15, (int64_t)a.n_rows - 1) * a.groups + first + N * U <= (int64_t)a.n_rows * a.groups;
            scale[t].load(a.scales, place[t].row * a.groups, place[t].scales, first, a.groups, inside);
            if constexpr (ZERO) zero[t].load(a.zeros, place[t].row * a.groups, place[t].scales, first, a.groups, inside);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int chunk = min(chunk0 + u, last);
#pragma unroll
            for (int t = 0; t < RT; t++) {
                const uint8_t *codes = a.codes + place[t].row * a.pitch + (int64_t)chunk * 64;
                words[u][t] = *reinterpret_cast<const uint4_t *>(codes + (chunk == last ? place[t].codes_last : place[t].codes));
            }
        }
    }
    // of the chunk's g-th group
    static __device__ __forceinline__ float of(const Scales<S, N * U> &s, int shift, int u, int g)
    {
        if constexpr (GM < 4 || U == 1) return to_f32(s.v[u * N + g]);
        const float own = to_f32(s.v[u]), of_two = to_f32(s.v[u / 2]), of_all = to_f32(s.v[0]);  // (chosen from as values: from among places in the array, it would be in memory)
        return shift == 7 ? own : shift == 8 ? of_two : of_all;
    }
};

// The x that a lane hands to the matrix instruction, a slot's (of each set) or none: then zeros, which lie in front of x in LDS.  On the side of the
// sums a lane's i-th one is of slot quarter + 4 i of the set and of row lane % 16 of the tile.
extern __shared__ uint4_t lds[];
constexpr int kZeros = 256;              // bytes
constexpr int kStagePad = 8;             // values between slots in LDS: sixteen slots' 16 bytes at one column are of different banks
template <int SETS, int NR> struct Side {
    uint32_t at[SETS], all[SETS];
    __device__ __forceinline__ void set(int slots, int stride)
    {
        const int lane = threadIdx.x % kWave, slot = (lane & 15) / 4 + 4 * (lane & 3);
#pragma unroll
        for (int k = 0; k < SETS; k++) {
            const bool mine = (lane & 3) < NR && 16 * k + slot < slots;
            at[k] = mine ? (uint32_t)(kZeros + (16 * k + slot) * stride * 2 + (lane >> 4) * 16) : 0u;
            all[k] = mine ? ~0u : 0u;
        }
    }
    __device__ __forceinline__ uint4_t x(int k, uint32_t byte, int piece) const
    {
        return *reinterpret_cast<const uint4_t *>(reinterpret_cast<const char *>(lds) + (at[k] + (byte & all[k])) + piece * 64);
    }
};
__device__ __forceinline__ void clear_zeros()
{
    if (threadIdx.x < kZeros / 16) lds[threadIdx.x] = uint4_t{0, 0, 0, 0};
}

// Adds what a batch's chunks contribute; byte: of the first one's columns behind a slot's start.  T: of x.
template <typename T, typename S, bool ZERO, int GM, int SETS, int NR, int RT, int U>
__device__ __forceinline__ void add_batch(const Batch<S, ZERO, GM, RT, U> &b, const Side<SETS, NR> &side, int shift, uint32_t byte, Constants constants, float (&acc)[RT][SETS][NR])
{
    constexpr bool kCodes = sizeof(T) == 4;  // codes as they are, not as 16 + q
    // A zero point is taken off as a bf16, which is all of it where it is a code.  The rest of it, if any, as further bf16 numbers where groups are of 32 columns, or else by the group's
    // sum of x, in fp32; us, fp32: 16 x 16384 x 4096 with groups of 32 and fp16 zero points 47 as numbers, 172 by the sum (registers); 16 x 20000 x 4096 with groups of 128 76 and 68.
    // (Not by a branch for zero points that are no codes: behind one that it put between a matrix instruction and what reads the result, the compiler left out wait states.)
    constexpr int kZeroParts = GM > 1 || std::is_same_v<S, bf16> ? 1 : std::is_same_v<S, f16> ? 2 : 3;
    constexpr bool kTaken = !kCodes || (ZERO && GM > 1 && !std::is_same_v<S, bf16>);
    using MT = std::conditional_t<kCodes, bf16, T>;
    using C = Cores<MT>;
#pragma unroll
    for (int u = 0; u < U; u++) {
        uint4_t words[RT];
#pragma unroll
        for (int t = 0; t < RT; t++) {
            words[t] = b.words[u][t];
            transpose_quarters(words[t]);
        }
#pragma unroll
        for (int g = 0; g < 4 / GM; g++) {
            uint4_t v[GM][SETS];
            float4_t taken[SETS];  // what the 16, and a zero point of 8, add to a group's sum; with zero points: the group's sum of x
#pragma unroll
            for (int k = 0; k < SETS; k++) {
                taken[k] = float4_t{0, 0, 0, 0};
                constexpr uint32_t kept = ZERO ? C::kOne : C::kMinus24;
#pragma unroll
                for (int j = 0; j < GM; j++) {
                    v[j][k] = side.x(k, byte + u * 256, g * GM + j);
                    if constexpr (kTaken) taken[k] = C::mul(v[j][k], uint4_t{kept, kept, kept, kept}, taken[k]);
                }
            }
#pragma unroll
            for (int t = 0; t < RT; t++) {
                const float f = b.of(b.scale[t], shift, u, g), zero = ZERO ? b.of(b.zero[ZERO ? t : 0], shift, u, g) : 8.0f;
                float off = -16.0f - zero;
                float4_t sum[SETS];
                if constexpr (kCodes) {
                    uint32_t minus[ZERO ? kZeroParts : 1];
                    float rest = -zero;
#pragma unroll
                    for (uint32_t &part : minus) {
                        part = __builtin_bit_cast(uint32_t, __builtin_convertvector(float2_t{rest, rest}, bf16x2_t));
                        rest -= __uint_as_float(part & 0xffff0000u);
                    }
                    off = rest;
#pragma unroll
                    for (int k = 0; k < SETS; k++) sum[k] = float4_t{0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < GM; j++) {
#pragma unroll
                        for (int i = (int)(sizeof(minus) / 4) - 1; i >= 0; i--)  // (the small ones while the sum is small)
#pragma unroll
                            for (int k = 0; k < SETS; k++) sum[k] = C::mul(v[j][k], uint4_t{minus[i], minus[i], minus[i], minus[i]}, sum[k]);
                        const uint4_t w = codes_of(words[t][g * GM + j]);
#pragma unroll
                        for (int k = 0; k < SETS; k++) sum[k] = C::mul(v[j][k], w, sum[k]);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < SETS; k++) sum[k] = ZERO ? float4_t{0, 0, 0, 0} : taken[k];
#pragma unroll
                    for (int j = 0; j < GM; j++) {
                        const uint4_t w = numbers_of<MT>(words[t][g * GM + j], constants);
#pragma unroll
                        for (int k = 0; k < SETS; k++) sum[k] = C::mul(v[j][k], w, sum[k]);
                    }
                }
#pragma unroll
                for (int k = 0; k < SETS; k++)
#pragma unroll
                    for (int i = 0; i < NR; i++) acc[t][k][i] += f * (ZERO && kTaken ? sum[k][i] + off * taken[k][i] : sum[k][i]);
            }
        }
    }
}

// x of 8 << log_eights columns from column `from` on, for `vectors` vectors, on its way into LDS: loaded (begin), later stored (end).
constexpr int kStagedEights = 4;         // for a thread, at most
template <typename T> struct Staging {
    static constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
    Staged<T> staged[kStagedEights];
    __device__ __forceinline__ void begin(const Q4Product &p, int64_t vector0, int vectors, int from, int log_eights)
    {
        if (p.a.n_cols < 8) return;
        const T *x = static_cast<const T *>(p.x) + vector0 * p.ldx;
#pragma unroll
        for (int e = 0; e < kStagedEights; e++)
            if ((int)(e * blockDim.x) < vectors << log_eights) {
                const int i = threadIdx.x + e * blockDim.x, v = min(i >> log_eights, vectors - 1);
                const int col = min(from + (i & ((1 << log_eights) - 1)) * 8, p.a.n_cols - 8);
                staged[e].v.load(x + v * p.ldx + col);
            }
    }
    __device__ __forceinline__ void end(const Q4Product &p, int64_t vector0, int vectors, int from, int log_eights, uint16_t *x, int stride)
    {
#pragma unroll
        for (int e = 0; e < kStagedEights; e++) {
            const int i = threadIdx.x + e * blockDim.x, v = i >> log_eights, eight = i & ((1 << log_eights) - 1);
            if (v < vectors) {
                const int col = from + eight * 8;
                if (col + 8 > p.a.n_cols) {
                    staged[e].v.clear();
                    if (col < p.a.n_cols) staged[e].v.load_first(static_cast<const T *>(p.x) + (vector0 + v) * p.ldx + col, p.a.n_cols - col);
                }
                staged[e].store(reinterpret_cast<uint32_t *>(x) + (v * kParts * stride) / 2 + eight * 4, stride / 2);
            }
        }
    }
};

// The wavefronts' sums of one tile of 16 rows each are added over the column_waves by LDS and written: [wave][k][i][lane].
template <typename T, typename S, int SETS, int NR>
__device__ __forceinline__ void add_up_and_write(const Q4Product &p, const float (&acc)[SETS][NR], float *sums, int64_t first_row, int log_row_waves, int rows_apart, int64_t vector0,
                                                 int vectors)
{
    constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, column_waves = blockDim.x / kWave >> log_row_waves, row_waves = 1 << log_row_waves;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SETS; k++)
#pragma unroll
        for (int i = 0; i < NR; i++) sums[((wave * SETS + k) * NR + i) * kWave + lane] = acc[k][i];
    __syncthreads();
    const int outputs = 16 * row_waves * vectors;
    for (int i0 = 0; i0 < outputs; i0 += blockDim.x) {
        const int i = i0 + threadIdx.x;
        const int v = i >> (4 + log_row_waves), rw = (i >> 4) & (row_waves - 1);
        const int64_t row = first_row + rw * rows_apart + (i & 15);
        const bool mine = i < outputs && row < p.a.n_rows;
        float sum = 0;
        if (mine)
            for (int part = 0; part < kParts; part++) {
                const int slot = v * kParts + part;
                float one = 0;
                for (int w = 0; w < column_waves; w++)
                    one += sums[(((w * row_waves + rw) * SETS + (slot >> 4)) * NR + (slot >> 2 & 3)) * kWave + (slot & 3) * 16 + (i & 15)];
                sum += one;
            }
        uint64_t again = __ballot(mine && !(fabsf(sum) < INFINITY));
        while (again) {
            const int from = __builtin_ctzll(again);
            again &= again - 1;
            const int j = i0 + (int)(threadIdx.x - lane) + from;
            const float exact = by_definition<T, S>(p, first_row + ((j >> 4) & (row_waves - 1)) * rows_apart + (j & 15), vector0 + (j >> (4 + log_row_waves)));
            if (lane == from) sum = exact;
        }
        if (mine) static_cast<T *>(p.y)[(vector0 + v) * p.ldy + row] = from_f32<T>(sum);
    }
}

// A workgroup of row_waves * column_waves wavefronts takes row_waves * RT * 16 rows.  In a step each column_wave takes U chunks of 128 columns; x of
// the step lies in LDS, that of the next one, and its codes and scales, are on their way into registers meanwhile.  The column_waves are added up at the end.
// GM: pieces of 32 columns that share a scale (4: 128 columns and more).  SETS: slots / 16, NR: slots of a set / 4, each rounded up (NR to 1 or 4).
// Bound: latency.  One vector: a chain of load, barrier, sum; 4096 x 4096 bf16 4 to 6 us.  Many: 204 to 256 registers leave one workgroup a compute unit; 48 x 131072 x 4096 fp16 139 to 146
// us (298 MB, 350 TFLOP/s; vector unit 45 %, matrix cores 20 % busy).  Held to 128 registers it spills (173).
constexpr int kMostSlots = 64;
constexpr int kStageBytes = 140 * 1024;  // of LDS, at most
constexpr int kThreads = 512;
template <typename T, typename S, bool ZERO, int GM, int SETS, int NR, int RT, int U>
__global__ __launch_bounds__(kThreads) void k_q4_mv(Q4Product p, int32_t per_pass, int32_t log_row_waves)
{
    using MT = std::conditional_t<sizeof(T) == 4, bf16, T>;
    constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const int row_waves = 1 << log_row_waves, column_waves = waves >> log_row_waves, row_wave = wave & (row_waves - 1), column_wave = wave >> log_row_waves;
    const int64_t vector0 = (int64_t)blockIdx.y * per_pass;
    const int vectors = (int)min((int64_t)per_pass, p.vectors - vector0), slots = vectors * kParts;
    const int64_t first_row = (int64_t)blockIdx.x * row_waves * (16 * RT), row0 = first_row + row_wave * (16 * RT);
    Place<S> place[RT];
#pragma unroll
    for (int t = 0; t < RT; t++) place[t].at(p.a, row0 + 16 * t);
    const int chunks = (p.a.n_cols + 127) / 128;
    const int step_chunks = column_waves * U, log_eights = __builtin_ctz(step_chunks) + 4;  // (a power of two)
    const int steps = (chunks + step_chunks - 1) >> (log_eights - 4);
    const int stride = step_chunks * 128 + kStagePad, buffer = per_pass * kParts * stride;  // values of a slot and of all in LDS
    uint16_t *const x0 = reinterpret_cast<uint16_t *>(lds) + kZeros / 2, *const x1 = x0 + buffer;
    const uint32_t byte0 = column_wave * U * 256, byte1 = byte0 + buffer * 2;
    Side<SETS, NR> side;
    side.set(slots, stride);
    const Constants constants = Constants::of<Cores<MT>>();
    clear_zeros();

    float acc[RT][SETS][NR] = {};
    Staging<T> staging;
    Batch<S, ZERO, GM, RT, U> a, b;
    staging.begin(p, vector0, vectors, 0, log_eights);
    a.load(p.a, place, column_wave * U);
    for (int step = 0; step < steps; step += 2) {  // (a step's loads are issued before those of the step before are waited for: two sets of registers in turn)
        staging.end(p, vector0, vectors, step * step_chunks * 128, log_eights, x0, stride);
        if (step + 1 < steps) {
            staging.begin(p, vector0, vectors, (step + 1) * step_chunks * 128, log_eights);
            b.load(p.a, place, (step + 1) * step_chunks + column_wave * U);
        }
        __syncthreads();
        add_batch<T>(a, side, p.a.shift, byte0, constants, acc);
        if (step + 1 < steps) {
            staging.end(p, vector0, vectors, (step + 1) * step_chunks * 128, log_eights, x1, stride);
            if (step + 2 < steps) {
                staging.begin(p, vector0, vectors, (step + 2) * step_chunks * 128, log_eights);
                a.load(p.a, place, (step + 2) * step_chunks + column_wave * U);
            }
            __syncthreads();
            add_batch<T>(b, side, p.a.shift, byte1, constants, acc);
        }
    }
#pragma unroll
    for (int t = 0; t < RT; t++) add_up_and_write<T, S>(p, acc[t], reinterpret_cast<float *>(lds), first_row + 16 * t, log_row_waves, 16 * RT, vector0, vectors);
}

// Many rows and few slots: x stays in LDS as a whole, and each wavefront walks through tiles of RT times 16 rows by itself, all columns of a tile after one
// another, the next U chunks always on their way: no barrier, and nothing to add up but the parts of an fp32 x.  Bound: HBM; 131072 x 4096 bf16, groups of 64, 57.4 us, 4.9 TB/s
// of 6 that such tiles can be read at (some 60 vector instructions for 16 rows x 128 columns, 28 % of the unit).
template <typename T, typename S, bool ZERO, int GM, int NR, int RT, int U>
__global__ __launch_bounds__(kThreads) void k_q4_mv_rows(Q4Product p)
{
    using MT = std::conditional_t<sizeof(T) == 4, bf16, T>;
    constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
    const int lane = threadIdx.x % kWave, waves = blockDim.x / kWave;
    const int vectors = (int)p.vectors, slots = vectors * kParts;
    const int chunks = (p.a.n_cols + 127) / 128, batches = (chunks + U - 1) / U;
    const int stride = (p.a.n_cols + 1023) / 1024 * 1024 + kStagePad;
    uint16_t *const x = reinterpret_cast<uint16_t *>(lds) + kZeros / 2;
    const int64_t tiles = ((int64_t)p.a.n_rows + 16 * RT - 1) / (16 * RT), apart = (int64_t)gridDim.x * waves;
    int64_t tile = (int64_t)blockIdx.x * waves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    Side<1, NR> side;
    side.set(slots, stride);
    const Constants constants = Constants::of<Cores<MT>>();
    clear_zeros();

    Batch<S, ZERO, GM, RT, U> a, b;
    Place<S> place[RT];
    int64_t load_tile = tile;
    int load_batch = 0;
#pragma unroll
    for (int t = 0; t < RT; t++) place[t].at(p.a, (tile * RT + t) * 16);
    auto load = [&](Batch<S, ZERO, GM, RT, U> &to) {  // the next of this wavefront's batches (behind the last tile: the last row's again)
        to.load(p.a, place, load_batch * U);
        if (++load_batch == batches) {
            load_batch = 0;
            load_tile += apart;
#pragma unroll
            for (int t = 0; t < RT; t++) place[t].at(p.a, (load_tile * RT + t) * 16);
        }
    };
    load(a);
    for (int from = 0; from < stride - kStagePad; from += 1024) {  // (128 times eight columns; the rest of the last ones is beyond x's place)
        Staging<T> staging;
        staging.begin(p, 0, vectors, from, 7);
        staging.end(p, 0, vectors, from, 7, x + from, stride);
    }
    __syncthreads();
    float acc[RT][1][NR] = {};
    int batch = 0;
    auto step = [&](const Batch<S, ZERO, GM, RT, U> &now) {
        add_batch<T>(now, side, p.a.shift, batch * (U * 256), constants, acc);
        if (++batch < batches) return;
        batch = 0;
#pragma unroll
        for (int t = 0; t < RT; t++) {
            const int64_t first = (tile * RT + t) * 16, row = first + (lane & 15);
#pragma unroll
            for (int v = 0; v < 4 * NR / kParts; v++) {
                if (v >= vectors) break;
                float sum = 0;
#pragma unroll
                for (int part = 0; part < kParts; part++) sum += __shfl(acc[t][0][(v * kParts + part) / 4], (v * kParts + part) % 4 * 16 + (lane & 15));
                uint64_t again = __ballot(lane < 16 && row < p.a.n_rows && !(fabsf(sum) < INFINITY));
                while (again) {
                    const int from = __builtin_ctzll(again);
                    again &= again - 1;
                    const float exact = by_definition<T, S>(p, first + from, v);
                    if (lane == from) sum = exact;
                }
                if (lane < 16 && row < p.a.n_rows) static_cast<T *>(p.y)[v * p.ldy + row] = from_f32<T>(sum);
            }
#pragma unroll
            for (int i = 0; i < NR; i++) acc[t][0][i] = 0;
        }
        tile += apart;
    };
    while (tile < tiles) {
        load(b);
        step(a);
        if (tile >= tiles) break;
        load(a);
        step(b);
    }
}

// Which kernel, and its shape.  Measured, us (bf16, groups of 128, where nothing else is said), the shapes in the order RT, U, wavefronts, row_waves (rows: k_q4_mv_rows):
//   1 to 4 slots: where each wavefront of two workgroups a compute unit has tiles to walk through, rows; 131072 x 4096 53.5 (1 4 4 4: 55.4; groups of 64: 57.4 and 57.3).  Else few
//     row_waves, so that a column_wave's way is short: 4096 x 4096 1 4 8 1 5.5, with two row_waves 6.9.  Four chunks where that is all there are, or in several steps: fp32 8192 x 28672 1 4 8 2 35, 1 2 8 2 39.
//     Else two: groups of 64, 10000 x 7000 1 2 8 2 17.0, 1 4 8 2 20.3, 4000 x 5000 1 2 8 1 6.3, 1 4 8 1 7.6 (not best where steps of four come out even: 14336 x 4096 1 2 8 2 15.3, 1 4 8 2 13.3).  Short rows
//     leave eight wavefronts nothing to do: 1000 x 1000 1 2 4 1 3.3, 1 2 8 1 3.7.
//   5 to 16: 16 x 4096 x 4096 1 1 8 1 8.0, 1 2 8 2 9.1; fp32 5 x 10007 x 7001, groups of 32, 1 2 8 4 25.8, 1 2 8 2 30.4, 1 1 8 4 30.8 (with zero points 32.1, 37.3, 39.0); 12 x 40000 x 4096 1 2 4 4 31, 1 2 8 4 40.
//   more: as many column_waves as x of a step fits the threads' registers with, and with many rows none; 24 x 8192 x 8192 1 1 8 2 23.2, 2 1 8 2 30.8;
//     64 x 4096 x 4096 1 1 8 4 28.8, 1 1 8 8 44.6; 48 x 131072 x 4096, groups of 64, 2 1 8 8 138, 1 1 8 8 169; 64 x 32768 x 8192 1 1 8 8 90, 2 1 8 8 about twice that (registers).
//     Two tiles of three sets, four groups a chunk and zero points do not fit the registers (38 to 90 spilled): one; 48 x 20000 x 4096 bf16 47, two 105; 48 x 131072 x 4096 199, two 273.
template <typename T, typename S, bool ZERO, int GM> int launch_mv(const Q4Product &p, hipStream_t st)
{
    constexpr int kParts = sizeof(T) == 4 ? 3 : 1, kThreeSetTiles = ZERO && GM == 1 ? 1 : 2;
    const int per_pass = (int)std::min<int64_t>(kMostSlots / kParts, p.vectors);
    const int slots = per_pass * kParts, sets = (slots + 15) / 16;
    const int64_t tiles = (p.a.n_rows + 15) / 16, chunks = (p.a.n_cols + 127) / 128, passes = (p.vectors + per_pass - 1) / per_pass;
    const size_t whole_x = kZeros + ((chunks + 7) / 8 * 1024 + kStagePad) * 2 * slots;
    if (slots <= 4 && tiles >= 4096 && whole_x <= kStageBytes / 2) {
        auto kernel = k_q4_mv_rows<T, S, ZERO, GM, 1, 1, 4>;
        if (whole_x > 64 * 1024) HBP_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kStageBytes));
        kernel<<<512, kThreads, whole_x, st>>>(p);
        HBP_HIP(hipGetLastError());
        return HBP_OK;
    }
    int waves = 8, row_waves, rt = 1, u = 1;
    if (slots <= 4) {
        waves = chunks > 8 ? 8 : 4;
        row_waves = tiles >= 512 ? 2 : 1;
        const int64_t four = 4 * (waves / row_waves);  // chunks of a step with U = 4: of use where they are all there are, or where there are several steps
        u = (chunks > four / 2 && chunks <= four) || chunks >= 4 * four ? 4 : 2;
    } else if (sets == 1) {
        waves = tiles >= 2048 ? 4 : 8;
        row_waves = tiles > 512 ? 4 : 1;
        u = tiles > 512 ? 2 : 1;
    } else {
        row_waves = tiles >= 1024 ? 8 : 2;
        while (row_waves < 8 && (per_pass * (waves / row_waves) * 16 > kStagedEights * kThreads ||
                                 slots * (waves / row_waves * 128 + kStagePad) * 4 > kStageBytes - kZeros))
            row_waves *= 2;
        rt = tiles >= 1024 && sets < 4 ? (sets == 3 ? kThreeSetTiles : 2) : 1;
    }
    const int64_t step = waves / row_waves * u, steps = (chunks + step - 1) / step;
    const size_t bytes = std::max<size_t>(kZeros + (steps > 1 ? 2 : 1) * slots * (step * 128 + kStagePad) * 2, (size_t)waves * sets * (slots <= 4 ? 1 : 4) * kWave * 4);
    if (bytes > kStageBytes || per_pass * step * 16 > kStagedEights * waves * kWave) return HBP_ERR_INTERNAL;  // (cannot be, by the above)
    constexpr int64_t kPasses = 32768;  // of one launch: the grid's second dimension ends at 65535
    for (int64_t first = 0; first < passes; first += kPasses) {
        Q4Product q = p;
        q.x = static_cast<const T *>(p.x) + first * per_pass * p.ldx;
        q.y = static_cast<T *>(p.y) + first * per_pass * p.ldy;
        q.vectors = std::min(p.vectors - first * per_pass, kPasses * per_pass);
        const dim3 grid((unsigned)((tiles + rt * row_waves - 1) / (rt * row_waves)), (unsigned)((q.vectors + per_pass - 1) / per_pass));
        const int rc = [&](auto kernel) -> int {
            if (bytes > 64 * 1024) HBP_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kStageBytes));
            kernel<<<grid, waves * kWave, bytes, st>>>(q, per_pass, __builtin_ctz(row_waves));
            HBP_HIP(hipGetLastError());
            return HBP_OK;
        }(slots <= 4  ? (u == 4 ? k_q4_mv<T, S, ZERO, GM, 1, 1, 1, 4> : k_q4_mv<T, S, ZERO, GM, 1, 1, 1, 2>)
          : sets == 1 ? (u == 2 ? k_q4_mv<T, S, ZERO, GM, 1, 4, 1, 2> : k_q4_mv<T, S, ZERO, GM, 1, 4, 1, 1>)
          : sets == 2 ? (rt == 2 ? k_q4_mv<T, S, ZERO, GM, 2, 4, 2, 1> : k_q4_mv<T, S, ZERO, GM, 2, 4, 1, 1>)
          : sets == 3 ? (rt == 2 ? k_q4_mv<T, S, ZERO, GM, 3, 4, kThreeSetTiles, 1> : k_q4_mv<T, S, ZERO, GM, 3, 4, 1, 1>)
                      : k_q4_mv<T, S, ZERO, GM, 4, 4, 1, 1>);
        if (rc != HBP_OK) return rc;
    }
    return HBP_OK;
}

template <typename T, bool ZERO> int launch_q4_mv(const Q4Product &p, hipStream_t st)
{
    return by_type(p.scale_type, [&](auto s) -> int {
        using S = decltype(s);
        return p.a.shift == 5 ? launch_mv<T, S, ZERO, 1>(p, st) : p.a.shift == 6 ? launch_mv<T, S, ZERO, 2>(p, st) : launch_mv<T, S, ZERO, 4>(p, st);
    });
}

}  // namespace
}  // namespace hbp
