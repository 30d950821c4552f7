// What the operators beside the sparse products share: value types, loads of eight values, sums over wavefronts and workgroups.
#pragma once

#include "hbp_internal.h"

#include <type_traits>

namespace hbp {

using f16 = _Float16;
using bf16 = __bf16;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(f16 v) { return (float)v; }
__device__ __forceinline__ float to_f32(bf16 v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_f32(float v) { return (T)v; }  // to nearest, ties to even

// Eight values at an address of which only the value's own alignment is known: whole loads of 16 bytes all the same, which gfx950
// serves from any address.
typedef uint32_t words_at_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t words_at_4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T> struct Eight {
    static constexpr int kWords = sizeof(T) * 2;
    using words_t = std::conditional_t<sizeof(T) == 2, words_at_2, words_at_4>;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < kWords / 4; i++) {
            const words_t v = *reinterpret_cast<const words_t *>(p + 16 / sizeof(T) * i);
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
    }
    __device__ __forceinline__ void store(T *p) const
    {
#pragma unroll
        for (int i = 0; i < kWords / 4; i++) {
            words_t v;
            v.x = w[4 * i]; v.y = w[4 * i + 1]; v.z = w[4 * i + 2]; v.w = w[4 * i + 3];
            *reinterpret_cast<words_t *>(p + 16 / sizeof(T) * i) = v;
        }
    }
    // value i as a float; bit for bit a T where it came from one
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(w[i]);
        } else {
            const uint16_t bits = (uint16_t)(w[i / 2] >> (i & 1) * 16);
            return to_f32(__builtin_bit_cast(T, bits));
        }
    }
    __device__ __forceinline__ void set(int i, float v)
    {
        if constexpr (sizeof(T) == 4) {
            w[i] = __float_as_uint(v);
        } else {
            const uint32_t bits = __builtin_bit_cast(uint16_t, from_f32<T>(v));
            w[i / 2] = (i & 1) ? (w[i / 2] & 0xffffu) | bits << 16 : bits;  // (in ascending order of i)
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < kWords; i++) w[i] = 0;
    }
    // The compiler no longer knows these values: it cannot use again what it has made of them so far.
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int i = 0; i < kWords; i++) asm("" : "+v"(w[i]));
    }
    // the first `n` of eight (n >= 8: all); the others are zero, and not read
    __device__ __forceinline__ void load_first(const T *p, int64_t n)
    {
        if (n >= 8) {
            load(p);
        } else {
            clear();
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (i < n) set_bits(i, p[i]);
        }
    }
    __device__ __forceinline__ void store_first(T *p, int64_t n) const
    {
        if (n >= 8) {
            store(p);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (i < n) p[i] = bits_of(i);
        }
    }
    __device__ __forceinline__ void set_bits(int i, T v)
    {
        if constexpr (sizeof(T) == 4) w[i] = __builtin_bit_cast(uint32_t, v);
        else w[i / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, v) << (i & 1) * 16;
    }
    __device__ __forceinline__ T bits_of(int i) const
    {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, w[i]);
        else return __builtin_bit_cast(T, (uint16_t)(w[i / 2] >> (i & 1) * 16));
    }
};

// op over the LANES (8 to 64) neighbouring lanes that a lane is among, the same result in all of them, by lane exchanges of the vector unit alone (quads, halves of
// rows, rows, quarters, halves).
template <int LANES = kWave, typename V, typename F> __device__ __forceinline__ V wave_reduce(V v, F op)
{
    static_assert(sizeof(V) == 4 && LANES >= 8, "");
    auto dpp = [&](auto control) {
        return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(control)::value, 0xf, 0xf, true));
    };
    v = op(v, dpp(std::integral_constant<int, 0xb1>()));   // quad_perm 1 0 3 2
    v = op(v, dpp(std::integral_constant<int, 0x4e>()));   // quad_perm 2 3 0 1
    v = op(v, dpp(std::integral_constant<int, 0x141>()));  // row_half_mirror
    if constexpr (LANES >= 16) v = op(v, dpp(std::integral_constant<int, 0x140>()));  // row_mirror
    if constexpr (LANES >= 32) {
        const uint32_t w = __builtin_bit_cast(uint32_t, v);
        auto a = __builtin_amdgcn_permlane16_swap(w, w, false, false);
        v = op(__builtin_bit_cast(V, (uint32_t)a[0]), __builtin_bit_cast(V, (uint32_t)a[1]));
    }
    if constexpr (LANES >= 64) {
        const uint32_t w = __builtin_bit_cast(uint32_t, v);
        auto a = __builtin_amdgcn_permlane32_swap(w, w, false, false);
        v = op(__builtin_bit_cast(V, (uint32_t)a[0]), __builtin_bit_cast(V, (uint32_t)a[1]));
    }
    return v;
}
__device__ __forceinline__ float wave_sum(float v)
{
    return wave_reduce(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v)  // (passes over NaN)
{
    return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    return wave_reduce(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

// Sums of N values over the THREADS of a workgroup, the same in every thread; with THREADS below 64, over each THREADS neighbouring lanes. `slots`: LDS, THREADS / 64 * N
// floats, that no other wavefront still reads (two calls in a row need two arrays).
template <int N, int THREADS> __device__ __forceinline__ void block_sums(float (&v)[N], float *slots)
{
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = wave_reduce<(THREADS < kWave ? THREADS : kWave)>(v[i], [](float a, float b) { return a + b; });
    if constexpr (THREADS > kWave) {
        const int wave = threadIdx.x / kWave;
        if (threadIdx.x % kWave == 0)
#pragma unroll
            for (int i = 0; i < N; i++) slots[wave * N + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; i++) {
            v[i] = 0;
#pragma unroll
            for (int k = 0; k < THREADS / kWave; k++) v[i] += slots[k * N + i];
        }
    }
}

// An error that an earlier call of this thread has left is reported before anything is launched.
inline int earlier_error()
{
    HBP_HIP(hipGetLastError());
    return HBP_OK;
}

inline bool is_type(int type) { return type == HBP_F32 || type == HBP_F16 || type == HBP_BF16; }
inline int64_t type_bytes(int type) { return type == HBP_F32 ? 4 : 2; }
inline bool aligned(const void *p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

// f(a value of the C++ type that `type` names)
template <typename F> int by_type(int type, F f)
{
    switch (type) {
    case HBP_F32: return f(float());
    case HBP_F16: return f(f16());
    case HBP_BF16: return f(bf16());
    default: return HBP_ERR_INVALID_ARGUMENT;
    }
}

}  // namespace hbp
