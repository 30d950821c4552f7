// Matrices held in 4 bits with group scales: packing, and products with a few vectors (hbp_q4_pack, hbp_q4_unpack, hbp_q4_mv, hbp_q4_mv_t).
#include "hbp_q4.h"

namespace hbp {
namespace {

template <typename S> __device__ __forceinline__ float scale_of(const Q4 &a, int64_t row, int group)
{
    return to_f32(static_cast<const S *>(a.scales)[row * a.groups + group]);
}
template <typename S> __device__ __forceinline__ float zero_of(const Q4 &a, int64_t row, int group)
{
    return a.zeros ? to_f32(static_cast<const S *>(a.zeros)[row * a.groups + group]) : 8.0f;
}

// Packing: a lane takes eight columns, the group's 4 to 64 lanes exchange its extremes.
template <typename T, typename S> __global__ __launch_bounds__(256) void k_q4_pack(Q4 a, const void *w_, int64_t ldw)
{
    const int64_t row = blockIdx.y + (int64_t)blockIdx.z * 32768;
    if (row >= a.n_rows) return;
    const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    const int64_t left = a.n_cols - col;
    Eight<T> w;
    w.clear();
    if (left > 0) w.load_first(static_cast<const T *>(w_) + row * ldw + col, left);
    float low = 0.0f, high = 0.0f, odd = 0.0f;  // odd: NaN from a value that no scale fits
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float v = w.get(i);
        low = fminf(low, v);
        high = fmaxf(high, v);
        odd += v * 0.0f;
    }
    const int lanes = 1 << (a.shift - 3);
    for (int d = 1; d < lanes; d *= 2) {
        low = fminf(low, __shfl_xor(low, d));
        high = fmaxf(high, __shfl_xor(high, d));
        odd += __shfl_xor(odd, d);
    }
    if (col >= a.pitch * 2) return;
    constexpr float kLargest = std::is_same_v<S, f16> ? 65504.0f : std::is_same_v<S, bf16> ? 3.3895313892515355e38f : 3.4028234663852886e38f;
    const float wide = a.zeros ? (high - low) * (1.0f / 15.0f) : fmaxf(-low, high) * (1.0f / 7.0f);
    const S scale = from_f32<S>(fminf(wide, kLargest));
    const float s = to_f32(scale);
    const float zero = !a.zeros ? 8.0f : s == 0.0f ? 0.0f : rintf(-low / s);
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float q = s == 0.0f ? zero : rintf(w.get(i) / s + zero);
        const uint32_t code = odd == 0.0f ? (uint32_t)fminf(fmaxf(q, 0.0f), 15.0f) : 8u;
        if (i < left) word |= code << 4 * i;
    }
    *reinterpret_cast<uint32_t *>(const_cast<uint8_t *>(a.codes) + row * a.pitch + col / 2) = word;
    if ((threadIdx.x & (lanes - 1)) == 0 && left > 0) {
        const int64_t at = row * a.groups + (col >> a.shift);
        static_cast<S *>(const_cast<void *>(a.scales))[at] = odd == 0.0f ? scale : from_f32<S>(NAN);
        if (a.zeros) static_cast<S *>(const_cast<void *>(a.zeros))[at] = from_f32<S>(odd == 0.0f ? zero : 0.0f);
    }
}

template <typename T, typename S> __global__ __launch_bounds__(256) void k_q4_unpack(Q4 a, void *w, int64_t ldw)
{
    const int64_t row = blockIdx.y + (int64_t)blockIdx.z * 32768;
    const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    const int64_t left = a.n_cols - col;
    if (row >= a.n_rows || left <= 0) return;
    const uint32_t word = *reinterpret_cast<const uint32_t *>(a.codes + row * a.pitch + col / 2);
    const int group = (int)(col >> a.shift);
    const float s = scale_of<S>(a, row, group), zero = zero_of<S>(a, row, group);
    Eight<T> out;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        float v = ((float)(word >> 4 * i & 15u) - zero) * s;
        asm("" : "+v"(v));  // (an fp32 value, as everywhere: the compiler has an instruction that rounds the product to fp16 at once)
        out.set(i, v);
    }
    out.store_first(static_cast<T *>(w) + row * ldw + col, left);
}

// transposed: a thread per eight columns and vector, over a part of the rows; the parts are summed by a second kernel
template <typename T, typename S> __global__ __launch_bounds__(256) void k_q4_mv_t(Q4 a, const void *x_, int64_t ldx, float *partial, int64_t vectors, int64_t part)
{
    const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (col >= a.n_cols) return;
    const int64_t begin = blockIdx.y * part, end = min(begin + part, (int64_t)a.n_rows);
    const int group = (int)(col >> a.shift);
    for (int64_t m = 0; m < vectors; m++) {
        const T *x = static_cast<const T *>(x_) + m * ldx;
        float acc[8] = {};
        for (int64_t r = begin; r < end; r++) {
            const uint32_t word = *reinterpret_cast<const uint32_t *>(a.codes + r * a.pitch + col / 2);
            const float zero = zero_of<S>(a, r, group), u = scale_of<S>(a, r, group) * to_f32(x[r]);
#pragma unroll
            for (int i = 0; i < 8; i++) acc[i] += ((float)(word >> 4 * i & 15u) - zero) * u;
        }
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (col + i < a.n_cols) partial[(blockIdx.y * vectors + m) * a.n_cols + col + i] = acc[i];
    }
}

template <typename T> __global__ __launch_bounds__(256) void k_q4_sum_parts(const float *partial, int parts, int64_t vectors, int64_t n_cols, void *y, int64_t ldy)
{
    const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (col >= n_cols) return;
    for (int64_t m = blockIdx.y; m < vectors; m += gridDim.y) {
        float sum = 0;
        for (int p = 0; p < parts; p++) sum += partial[(p * vectors + m) * n_cols + col];
        static_cast<T *>(y)[m * ldy + col] = from_f32<T>(sum);
    }
}

int parts_of(const Q4 &a)
{
    const int64_t wide = (a.n_cols + 2047) / 2048, wanted = (1024 + wide - 1) / wide, most = (a.n_rows + 31) / 32;
    return (int)(wanted < most ? wanted : most);
}

int view(const hbp_q4_matrix_t *m, Q4 *a)
{
    if (!m || !m->codes || !m->scales || m->n_rows < 1 || m->n_cols < 1 || !is_type(m->scale_type)) return HBP_ERR_INVALID_ARGUMENT;
    if (m->n_rows > (int64_t(1) << 31) - 512 || m->n_cols > int64_t(1) << 28) return HBP_ERR_TOO_LARGE;
    int shift = 5;
    while (shift < 9 && (1 << shift) != m->group) shift++;
    const int64_t bytes = type_bytes(m->scale_type);
    if ((1 << shift) != m->group || !aligned(m->codes, 16) || !aligned(m->scales, bytes) || !aligned(m->zeros, bytes)) return HBP_ERR_INVALID_ARGUMENT;
    a->codes = static_cast<const uint8_t *>(m->codes); a->scales = m->scales; a->zeros = m->zeros;
    a->pitch = (m->n_cols + 31) / 32 * 16;
    a->n_rows = (int32_t)m->n_rows; a->n_cols = (int32_t)m->n_cols;
    a->groups = (int32_t)((m->n_cols + m->group - 1) >> shift); a->shift = shift;
    return HBP_OK;
}

// checks what both products share
int check_product(const hbp_q4_matrix_t *m, Q4 *a, int type, const void *x, int64_t ldx, int64_t n_x, const void *y, int64_t ldy, int64_t n_y, int64_t vectors)
{
    if (!is_type(type) || vectors < 0 || (vectors > 1 && (ldx < n_x || ldy < n_y))) return HBP_ERR_INVALID_ARGUMENT;
    if (vectors > (int64_t(1) << 31) - 512) return HBP_ERR_TOO_LARGE;
    if (vectors > 0 && (!x || !y || !aligned(x, type_bytes(type)) || !aligned(y, type_bytes(type)))) return HBP_ERR_INVALID_ARGUMENT;
    (void)m; (void)a;
    return HBP_OK;
}

}  // namespace
}  // namespace hbp

extern "C" {

int hbp_q4_pack(const hbp_q4_matrix_t *m, int type, const void *w, int64_t ldw, void *stream)
{
    using namespace hbp;
    Q4 a;
    int rc = view(m, &a);
    if (rc != HBP_OK) return rc;
    if (!is_type(type) || !w || !aligned(w, type_bytes(type)) || (m->n_rows > 1 && ldw < m->n_cols)) return HBP_ERR_INVALID_ARGUMENT;
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    const dim3 grid((unsigned)((a.pitch * 2 + 2047) / 2048), (unsigned)(a.n_rows < 32768 ? a.n_rows : 32768), (unsigned)((a.n_rows + 32767) / 32768));
    return by_type(type, [&](auto t) -> int {
        return by_type(m->scale_type, [&](auto s) -> int {
            k_q4_pack<decltype(t), decltype(s)><<<grid, 256, 0, (hipStream_t)stream>>>(a, w, ldw);
            HBP_HIP(hipGetLastError());
            return HBP_OK;
        });
    });
}

int hbp_q4_unpack(const hbp_q4_matrix_t *m, int type, void *w, int64_t ldw, void *stream)
{
    using namespace hbp;
    Q4 a;
    int rc = view(m, &a);
    if (rc != HBP_OK) return rc;
    if (!is_type(type) || !w || !aligned(w, type_bytes(type)) || (m->n_rows > 1 && ldw < m->n_cols)) return HBP_ERR_INVALID_ARGUMENT;
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    const dim3 grid((unsigned)((a.pitch * 2 + 2047) / 2048), (unsigned)(a.n_rows < 32768 ? a.n_rows : 32768), (unsigned)((a.n_rows + 32767) / 32768));
    return by_type(type, [&](auto t) -> int {
        return by_type(m->scale_type, [&](auto s) -> int {
            k_q4_unpack<decltype(t), decltype(s)><<<grid, 256, 0, (hipStream_t)stream>>>(a, w, ldw);
            HBP_HIP(hipGetLastError());
            return HBP_OK;
        });
    });
}

int hbp_q4_mv(const hbp_q4_matrix_t *m, int type, const void *x, int64_t ldx, void *y, int64_t ldy, int64_t vectors, void *stream)
{
    using namespace hbp;
    Q4 a;
    int rc = view(m, &a);
    if (rc == HBP_OK) rc = check_product(m, &a, type, x, ldx, m->n_cols, y, ldy, m->n_rows, vectors);
    if (rc != HBP_OK || vectors == 0) return rc;
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    const Q4Product p{a, x, y, ldx, ldy, vectors, m->scale_type};
    hipStream_t st = (hipStream_t)stream;
    if (a.zeros) return type == HBP_F32 ? launch_q4_mv_f32_zeros(p, st) : type == HBP_F16 ? launch_q4_mv_f16_zeros(p, st) : launch_q4_mv_bf16_zeros(p, st);
    return type == HBP_F32 ? launch_q4_mv_f32(p, st) : type == HBP_F16 ? launch_q4_mv_f16(p, st) : launch_q4_mv_bf16(p, st);
}

int hbp_q4_mv_t_workspace(const hbp_q4_matrix_t *m, int64_t vectors, size_t *bytes)
{
    using namespace hbp;
    Q4 a;
    const int rc = view(m, &a);
    if (rc != HBP_OK) return rc;
    if (!bytes || vectors < 0) return HBP_ERR_INVALID_ARGUMENT;
    *bytes = (size_t)parts_of(a) * (size_t)vectors * (size_t)a.n_cols * sizeof(float);
    return HBP_OK;
}

int hbp_q4_mv_t(const hbp_q4_matrix_t *m, int type, const void *x, int64_t ldx, void *y, int64_t ldy, int64_t vectors, void *workspace,
                size_t workspace_bytes, void *stream)
{
    using namespace hbp;
    Q4 a;
    size_t need = 0;
    int rc = view(m, &a);
    if (rc == HBP_OK) rc = check_product(m, &a, type, x, ldx, m->n_rows, y, ldy, m->n_cols, vectors);
    if (rc == HBP_OK) rc = hbp_q4_mv_t_workspace(m, vectors, &need);
    if (rc != HBP_OK || vectors == 0) return rc;
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return HBP_ERR_INVALID_ARGUMENT;
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    const int parts = parts_of(a);
    const int64_t part = (a.n_rows + parts - 1) / parts;
    const unsigned wide = (unsigned)((a.n_cols + 2047) / 2048);
    float *partial = static_cast<float *>(workspace);
    return by_type(type, [&](auto t) -> int {
        return by_type(m->scale_type, [&](auto s) -> int {
            k_q4_mv_t<decltype(t), decltype(s)><<<dim3(wide, parts), 256, 0, (hipStream_t)stream>>>(a, x, ldx, partial, vectors, part);
            HBP_HIP(hipGetLastError());
            k_q4_sum_parts<decltype(t)><<<dim3((unsigned)((a.n_cols + 255) / 256), (unsigned)(vectors < 64 ? vectors : 64)), 256, 0, (hipStream_t)stream>>>(
                partial, parts, vectors, a.n_cols, y, ldy);
            HBP_HIP(hipGetLastError());
            return HBP_OK;
        });
    });
}

}  // extern "C"
