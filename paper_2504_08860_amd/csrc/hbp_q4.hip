// Matrices held in 4 bits with group scales: packing, and products with a few vectors (hbp_q4_pack, hbp_q4_unpack, hbp_q4_mv, hbp_q4_mv_t).
#include "hbp_q4.h"

#include <algorithm>

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

// Extremes over the 4 to 64 lanes of a group: over quads and rows of sixteen by the vector unit's own lane exchanges.
template <typename F> __device__ __forceinline__ float group_reduce(float v, int lanes, F op)
{
    auto dpp = [&](auto control) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(control)::value, 0xf, 0xf, true));
    };
    v = op(v, dpp(std::integral_constant<int, 0xb1>()));   // quad_perm 1 0 3 2
    v = op(v, dpp(std::integral_constant<int, 0x4e>()));   // quad_perm 2 3 0 1
    if (lanes > 4) v = op(v, dpp(std::integral_constant<int, 0x141>()));  // row_half_mirror
    if (lanes > 8) v = op(v, dpp(std::integral_constant<int, 0x140>()));  // row_mirror
    for (int d = 16; d < lanes; d *= 2) v = op(v, __shfl_xor(v, d));
    return v;
}

// Packing: a lane takes eight columns of kPackRows rows, whose loads are all on their way at once.  The code is that of the quotient, but a product with the
// reciprocal, off by a few last bits, gives the same one unless it lies next to a half.  Bound: HBM; 8192 x 8192 bf16 46 to 51 us (168 MB; 58 with the division, one row at a time).
constexpr int kPackRows = 4;
template <typename T, typename S> __global__ __launch_bounds__(256) void k_q4_pack(Q4 a, const void *w_, int64_t ldw)
{
    const int64_t row0 = (blockIdx.y + (int64_t)blockIdx.z * 32768) * kPackRows;
    const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    const int64_t left = a.n_cols - col;
    Eight<T> w[kPackRows];
#pragma unroll
    for (int r = 0; r < kPackRows; r++) {
        w[r].clear();
        if (left > 0 && row0 + r < a.n_rows) w[r].load_first(static_cast<const T *>(w_) + (row0 + r) * ldw + col, left);
    }
    const int lanes = 1 << (a.shift - 3);
#pragma unroll
    for (int r = 0; r < kPackRows; r++) {
        float low = 0.0f, high = 0.0f, odd = 0.0f;  // odd: NaN from a value that no scale fits
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float v0 = w[r].get(i), v1 = w[r].get(i + 1);
            asm("v_min3_f32 %0, %1, %2, %0" : "+v"(low) : "v"(v0), "v"(v1));  // (fminf would make each value canonical first)
            asm("v_max3_f32 %0, %1, %2, %0" : "+v"(high) : "v"(v0), "v"(v1));
            odd = fmaf(v0, 0.0f, fmaf(v1, 0.0f, odd));
        }
        low = group_reduce(low, lanes, [](float x, float y) { return fminf(x, y); });
        high = group_reduce(high, lanes, [](float x, float y) { return fmaxf(x, y); });
        odd = group_reduce(odd, lanes, [](float x, float y) { return x + y; });
        const int64_t row = row0 + r;
        if (col >= a.pitch * 2 || row >= a.n_rows) continue;
        constexpr float kLargest = std::is_same_v<S, f16> ? 65504.0f : std::is_same_v<S, bf16> ? 3.3895313892515355e38f : 3.4028234663852886e38f;
        const float span = high - low;  // may be more than the largest number where a fifteenth of it is not
        const float wide = !a.zeros ? fmaxf(-low, high) * (1.0f / 7.0f) : span < INFINITY ? span * (1.0f / 15.0f) : high * (1.0f / 15.0f) - low * (1.0f / 15.0f);
        const S scale = from_f32<S>(fminf(wide, kLargest));
        const float s = to_f32(scale), inverse = s == 0.0f ? 0.0f : 1.0f / s;
        const float zero = !a.zeros ? 8.0f : s == 0.0f ? 0.0f : fminf(rintf(-low / s), 15.0f);
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float v = w[r].get(i);
            float q = fmaf(v, inverse, zero);
            if (!(fabsf(__builtin_amdgcn_fractf(q) - 0.5f) > 1e-4f)) q = s == 0.0f ? zero : v / s + zero;  // (also where the reciprocal is not finite)
            word |= (uint32_t)__builtin_amdgcn_fmed3f(rintf(q), 0.0f, 15.0f) << 4 * i;
        }
        if (odd != 0.0f) word = 0x88888888u;
        if (left < 8) word = left > 0 ? word & ((1u << 4 * left) - 1) : 0;
        *reinterpret_cast<uint32_t *>(const_cast<uint8_t *>(a.codes) + row * a.pitch + col / 2) = word;
        if ((threadIdx.x & (lanes - 1)) == 0 && left > 0) {
            const int64_t at = row * a.groups + (col >> a.shift);
            static_cast<S *>(const_cast<void *>(a.scales))[at] = odd == 0.0f ? scale : from_f32<S>(NAN);
            if (a.zeros) static_cast<S *>(const_cast<void *>(a.zeros))[at] = from_f32<S>(odd == 0.0f ? zero : 0.0f);
        }
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

// y = x W, the transposed product.  A lane takes C neighbouring columns (of one group) and adds (code - zero) * (scale x) row by row, in fp32, for up to M vectors
// (zero (scale x) as a sum of its own, taken off at the end, would be one fma for all C, and leave errors of its own size in a result that is much smaller where x is of
// one sign).  A workgroup has 64 C columns of a part of the rows, its wavefronts every eighth batch of ROWS rows; they are added up by LDS, the parts by a second kernel.
//
// Bound: vector instructions, 1.4 + M a weight (a conversion for each code, with zero points a subtraction more, and an fma for each vector), and their latency; us: 1 x 8192 x 8192 fp32 14 + 4 for the
// sum, 19 x 6001 x 4099 with zero points 30 + 4.5, 64 x 8192 x 8192 170 (51 TFLOP/s of the 79 that fp32 fma has here).  For the matrix cores the scale, which
// differs from row to row, would have to go into x, in two or three parts, once for each group of columns: not tried.
// As in the products, (code - zero) * (scale x) may be infinite where the sum is not: such results are computed again from the definition.
constexpr int kTransposedWaves = 8, kTransposedRows = 512;  // rows whose x lies in LDS at a time
// What a lane loads of ROWS rows.
template <typename S, bool ZERO, int C, int ROWS> struct Rows {
    uint32_t w[ROWS][C / 8];
    S scale[ROWS], zero[ZERO ? ROWS : 1];
    // at: bytes of the lane's columns in a row of codes; scale_at: of its group in a row of scales
    __device__ __forceinline__ void load(const Q4 &a, int64_t row0, int r, int rows, uint32_t at, uint32_t scale_at)
    {
        const int64_t apart = (int64_t)a.groups * (int64_t)sizeof(S);
        const uint8_t *codes = a.codes + (row0 + r) * a.pitch;
        const char *scales = static_cast<const char *>(a.scales) + (row0 + r) * apart, *zeros = static_cast<const char *>(a.zeros) + (row0 + r) * apart;
#pragma unroll
        for (int i = 0; i < ROWS; i++) {
            if constexpr (C == 16) {
                const uint2 two = *reinterpret_cast<const uint2 *>(codes + at);
                w[i][0] = two.x;
                w[i][1] = two.y;
            } else {
                w[i][0] = *reinterpret_cast<const uint32_t *>(codes + at);
            }
            scale[i] = *reinterpret_cast<const S *>(scales + scale_at);
            if constexpr (ZERO) zero[i] = *reinterpret_cast<const S *>(zeros + scale_at);
            const bool more = r + i + 1 < rows;  // (behind the last row it is read again: x is 0 there)
            codes += more ? a.pitch : 0;
            scales += more ? apart : 0;
            if constexpr (ZERO) zeros += more ? apart : 0;
        }
    }
    // x: of the first row's M vectors, then the next one's
    template <int M> __device__ __forceinline__ void add(const float *x, float (&acc)[M][C]) const
    {
#pragma unroll
        for (int i = 0; i < ROWS; i++) {
            const float s = to_f32(scale[i]) * (ZERO ? 1.0f : 16.0f), z = ZERO ? to_f32(zero[ZERO ? i : 0]) : 0.0f;
            float f[C], u[M];
            if constexpr (M % 4 == 0) {
#pragma unroll
                for (int m = 0; m < M; m += 4) {
                    const float4 four = *reinterpret_cast<const float4 *>(x + i * M + m);
                    u[m] = s * four.x; u[m + 1] = s * four.y; u[m + 2] = s * four.z; u[m + 3] = s * four.w;
                }
            } else if constexpr (M % 2 == 0) {
#pragma unroll
                for (int m = 0; m < M; m += 2) {
                    const float2 two = *reinterpret_cast<const float2 *>(x + i * M + m);
                    u[m] = s * two.x; u[m + 1] = s * two.y;
                }
            } else {
                u[0] = s * x[i];
            }
#pragma unroll
            for (int j = 0; j < C / 8; j++) {
                if constexpr (ZERO) {
                    const uint32_t even = w[i][j] & 0x0f0f0f0fu, odd = w[i][j] >> 4 & 0x0f0f0f0fu;
#pragma unroll
                    for (int b = 0; b < 4; b++) {
                        f[8 * j + 2 * b] = (float)(even >> 8 * b & 255u) - z;
                        f[8 * j + 2 * b + 1] = (float)(odd >> 8 * b & 255u) - z;
                    }
                } else {  // with 8 flipped a code is a number of four bits with a sign, of which the instruction makes (code - 8) / 16
                    const uint32_t even = w[i][j] ^ 0x88888888u, odd = even >> 4;
#pragma unroll
                    for (int b = 0; b < 4; b++) {
                        f[8 * j + 2 * b] = __builtin_amdgcn_cvt_off_f32_i4(even >> 8 * b & 255u);
                        f[8 * j + 2 * b + 1] = __builtin_amdgcn_cvt_off_f32_i4(odd >> 8 * b & 255u);
                    }
                }
            }
#pragma unroll
            for (int m = 0; m < M; m++)
#pragma unroll
                for (int c = 0; c < C; c++) acc[m][c] += f[c] * u[m];
        }
    }
};

template <typename T, typename S, bool ZERO, int M, int C, int ROWS>
__global__ __launch_bounds__(kTransposedWaves * kWave) void k_q4_mv_t(Q4 a, const void *x_, int64_t ldx, float *partial, int64_t vectors, int64_t part)
{
    extern __shared__ float4 lds4[];
    float *lds = reinterpret_cast<float *>(lds4);  // x of up to kTransposedRows rows of the part, [row][M]; then the sums of one vector, [wavefront][64 C]
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t vector0 = (int64_t)blockIdx.z * M;
    const int64_t part0 = (int64_t)blockIdx.y * part, end = min(part0 + part, (int64_t)a.n_rows);
    const int apart = (int)min(part, (int64_t)kTransposedRows);
    const T *x = static_cast<const T *>(x_);
    const int col = blockIdx.x * (kWave * C) + lane * C;
    const uint32_t at = min(col, (int)(a.pitch * 2) - C) / 2;  // (lanes behind the last column read its codes again)
    const uint32_t scale_at = min(col >> a.shift, a.groups - 1) * sizeof(S);
    float acc[M][C] = {};
    constexpr int kStep = kTransposedWaves * ROWS;
    for (int64_t row0 = part0; row0 < end; row0 += apart) {
        const int rows = (int)min((int64_t)apart, end - row0);
        Rows<S, ZERO, C, ROWS> one, two;
        int r = wave * ROWS;
        if (r < rows) one.load(a, row0, r, rows, at, scale_at);
        if (row0 > part0) __syncthreads();
#pragma unroll
        for (int m = 0; m < M; m++)
            for (int i = threadIdx.x; i < apart; i += blockDim.x) lds[i * M + m] = vector0 + m < vectors && i < rows ? to_f32(x[(vector0 + m) * ldx + row0 + i]) : 0.0f;
        __syncthreads();
        for (; r < rows; r += 2 * kStep) {  // (the next rows' loads are issued before this one's are waited for)
            if (r + kStep < rows) two.load(a, row0, r + kStep, rows, at, scale_at);
            one.template add<M>(lds + r * M, acc);
            if (r + kStep < rows) {
                if (r + 2 * kStep < rows) one.load(a, row0, r + 2 * kStep, rows, at, scale_at);
                two.template add<M>(lds + (r + kStep) * M, acc);
            }
        }
    }
#pragma unroll
    for (int m = 0; m < M; m++) {
        __syncthreads();
#pragma unroll
        for (int c = 0; c < C; c += 4)
            reinterpret_cast<float4 *>(lds)[(wave * (kWave * C) + lane * C + c) / 4] = float4{acc[m][c], acc[m][c + 1], acc[m][c + 2], acc[m][c + 3]};
        __syncthreads();
        if (vector0 + m < vectors)
            for (int c = threadIdx.x; c < kWave * C; c += blockDim.x) {
                float sum = 0;
#pragma unroll
                for (int w = 0; w < kTransposedWaves; w++) sum += lds[w * (kWave * C) + c];
                const int64_t k = (int64_t)blockIdx.x * (kWave * C) + c;
                if (k < a.n_cols) partial[((int64_t)blockIdx.y * vectors + vector0 + m) * a.n_cols + k] = sum;
            }
    }
}

// The parts' sum, in their order; a wavefront has 64 columns of one vector.
template <typename T, typename S> __global__ __launch_bounds__(256) void k_q4_sum_parts(Q4 a, const void *x_, int64_t ldx, const float *partial, int parts, int64_t vectors, void *y, int64_t ldy)
{
    const int lane = threadIdx.x % kWave;
    const int64_t m = (int64_t)blockIdx.y * 4 + threadIdx.x / kWave;
    if (m >= vectors) return;
    const int64_t col = (int64_t)blockIdx.x * kWave + lane;
    const bool mine = col < a.n_cols;
    float sum = 0;
    if (mine) {
        const float *at = partial + m * a.n_cols + col;
        const int64_t apart = vectors * a.n_cols;
        int i = 0;
        for (; i + 8 <= parts; i += 8) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; k++) v[k] = at[(i + k) * apart];
#pragma unroll
            for (int k = 0; k < 8; k++) sum += v[k];
        }
        for (; i < parts; i++) sum += at[i * apart];
    }
    uint64_t again = __ballot(mine && !(fabsf(sum) < INFINITY));
    while (again) {  // from the definition, by the whole wavefront
        const int from = __builtin_ctzll(again);
        again &= again - 1;
        const int64_t k = (int64_t)blockIdx.x * kWave + from;
        float exact = 0;
        for (int64_t r = lane; r < a.n_rows; r += kWave) {
            const float q = (float)(a.codes[r * a.pitch + k / 2] >> (k & 1) * 4 & 15);
            exact += scale_of<S>(a, r, (int)(k >> a.shift)) * (q - zero_of<S>(a, r, (int)(k >> a.shift))) * to_f32(static_cast<const T *>(x_)[m * ldx + r]);
        }
        exact = wave_sum(exact);
        if (lane == from) sum = exact;
    }
    if (mine) static_cast<T *>(y)[m * ldy + col] = from_f32<T>(sum);
}

// How a transposed product is cut: vectors, columns and rows at a time a lane takes, rows of a part, none of fewer rows than its wavefronts take at a time.
constexpr int kTransposedVectors[] = {1, 2, 4, 6, 8, 10};
struct TransposedShape {
    int m, c, rows;
    int64_t part, wide, parts;
};
TransposedShape transposed_shape(const Q4 &a, int64_t vectors)
{
    TransposedShape s;
    // Vectors at a time: an fma for each of a word's eight codes and each vector, and some 27 instructions besides (a conversion for each code, the word's and the scale's
    // loads): as few as may be in all.
    s.m = 1;
    int64_t least_cost = INT64_MAX;
    for (int m : kTransposedVectors) {
        const int64_t cost = (vectors + m - 1) / m * (27 + 9 * m);
        if (cost < least_cost) {
            least_cost = cost;
            s.m = m;
        }
    }
    s.c = s.m <= 2 ? 16 : 8;
    s.rows = s.m <= 2 ? 8 : 4;
    s.wide = (a.n_cols + kWave * s.c - 1) / (kWave * s.c);
    // Parts: a workgroup for each place on the chip (one of more than six vectors a compute unit, or two), or for several rounds of them; as many as
    // leave the fewest places empty in the last round.  19 x 6001 x 4099 in 432 workgroups 43.8 us, in 252 35.4.  (Ten vectors take 138 registers and more, of which one workgroup fits; eight without
    // zero points take 120, and two would fit, which is slower for one pass, 8 x 30000 x 2048 34.6 for 32.3, and faster for several, 64 x 8192 x 8192 142 for 170.)
    const int64_t passes = std::max<int64_t>((vectors + s.m - 1) / s.m, 1), least = 2 * s.rows * kTransposedWaves;
    const int64_t most = (a.n_rows + least - 1) / least, places = s.m > 6 ? 256 : 512, each = s.wide * passes;
    const int64_t first = std::max<int64_t>(places / each, 1);
    double fullest = 0;
    s.parts = 1;
    for (int64_t parts = first; parts < first + 8; parts++) {
        const int64_t all = std::min(parts, most) * each, rounds = (all + places - 1) / places;
        const double full = (double)all / (double)(rounds * places);
        if (full > fullest + 0.03) {
            fullest = full;
            s.parts = std::min(parts, most);
        }
    }
    s.part = ((a.n_rows + s.parts - 1) / s.parts + least - 1) / least * least;
    s.parts = (a.n_rows + s.part - 1) / s.part;
    return s;
}

int view(const hbp_q4_matrix_t *m, Q4 *a)
{
    if (!m || !m->codes || !m->scales || m->n_rows < 1 || m->n_cols < 1 || !is_type(m->scale_type)) return HBP_ERR_INVALID_ARGUMENT;
    if (m->n_rows > int64_t(1) << 30 || m->n_cols > int64_t(1) << 28) return HBP_ERR_TOO_LARGE;
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

constexpr int64_t kMostVectors = int64_t(1) << 24;  // (so that a workspace's bytes can be counted)
// Vectors of one pair of launches: the grids end at 65535 in the dimension of the passes and in that of the sum's fours of vectors.  The workspace is used again by the next pair.
int64_t vectors_at_once(const TransposedShape &s, int64_t vectors) { return std::min<int64_t>(vectors, 16384 * s.m); }

// checks what both products share
int check_product(int type, const void *x, int64_t ldx, int64_t n_x, const void *y, int64_t ldy, int64_t n_y, int64_t vectors)
{
    if (!is_type(type) || vectors < 0 || (vectors > 1 && (ldx < n_x || ldy < n_y))) return HBP_ERR_INVALID_ARGUMENT;
    if (vectors > kMostVectors) return HBP_ERR_TOO_LARGE;
    if (vectors > 0 && (!x || !y || !aligned(x, type_bytes(type)) || !aligned(y, type_bytes(type)))) return HBP_ERR_INVALID_ARGUMENT;
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
    const int64_t fours = ((int64_t)a.n_rows + kPackRows - 1) / kPackRows;
    const dim3 grid((unsigned)((a.pitch * 2 + 2047) / 2048), (unsigned)(fours < 32768 ? fours : 32768), (unsigned)((fours + 32767) / 32768));
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
    if (rc == HBP_OK) rc = check_product(type, x, ldx, m->n_cols, y, ldy, m->n_rows, vectors);
    if (rc != HBP_OK || vectors == 0) return rc;
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    hipStream_t st = (hipStream_t)stream;
    constexpr int32_t kRows = 1 << 26;  // of one launch: a grid counts its threads, up to sixteen for a row, in 32 bits
    const int64_t scale_bytes = type_bytes(m->scale_type) * a.groups;
    for (int64_t first = 0; first < m->n_rows; first += kRows) {
        Q4Product p{a, x, static_cast<char *>(y) + first * type_bytes(type), ldx, ldy, vectors, m->scale_type};
        p.a.codes += first * a.pitch;
        p.a.scales = static_cast<const char *>(a.scales) + first * scale_bytes;
        if (a.zeros) p.a.zeros = static_cast<const char *>(a.zeros) + first * scale_bytes;
        p.a.n_rows = (int32_t)std::min<int64_t>(m->n_rows - first, kRows);
        if (a.zeros) rc = type == HBP_F32 ? launch_q4_mv_f32_zeros(p, st) : type == HBP_F16 ? launch_q4_mv_f16_zeros(p, st) : launch_q4_mv_bf16_zeros(p, st);
        else rc = type == HBP_F32 ? launch_q4_mv_f32(p, st) : type == HBP_F16 ? launch_q4_mv_f16(p, st) : launch_q4_mv_bf16(p, st);
        if (rc != HBP_OK) return rc;
    }
    return HBP_OK;
}

int hbp_q4_mv_t_workspace(const hbp_q4_matrix_t *m, int64_t vectors, size_t *bytes)
{
    using namespace hbp;
    Q4 a;
    const int rc = view(m, &a);
    if (rc != HBP_OK) return rc;
    if (!bytes || vectors < 0) return HBP_ERR_INVALID_ARGUMENT;
    if (vectors > kMostVectors) return HBP_ERR_TOO_LARGE;
    const TransposedShape s = transposed_shape(a, vectors);
    *bytes = (size_t)s.parts * (size_t)vectors_at_once(s, vectors) * (size_t)a.n_cols * sizeof(float);
    return HBP_OK;
}

int hbp_q4_mv_t(const hbp_q4_matrix_t *m, int type, const void *x, int64_t ldx, void *y, int64_t ldy, int64_t vectors, void *workspace,
                size_t workspace_bytes, void *stream)
{
    using namespace hbp;
    Q4 a;
    size_t need = 0;
    int rc = view(m, &a);
    if (rc == HBP_OK) rc = check_product(type, x, ldx, m->n_rows, y, ldy, m->n_cols, vectors);
    if (rc == HBP_OK) rc = hbp_q4_mv_t_workspace(m, vectors, &need);
    if (rc != HBP_OK || vectors == 0) return rc;
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return HBP_ERR_INVALID_ARGUMENT;
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    const TransposedShape s = transposed_shape(a, vectors);
    float *partial = static_cast<float *>(workspace);
    hipStream_t st = (hipStream_t)stream;
    return by_type(type, [&](auto t) -> int {
        return by_type(m->scale_type, [&](auto scale) -> int {
            using T = decltype(t);
            using S = decltype(scale);
            for (int64_t first = 0; first < vectors;) {
                const int64_t count = vectors_at_once(s, vectors - first);
                const dim3 grid((unsigned)s.wide, (unsigned)s.parts, (unsigned)((count + s.m - 1) / s.m));
                const size_t x_bytes = (size_t)s.m * (s.part < kTransposedRows ? s.part : kTransposedRows) * 4, sum_bytes = (size_t)kTransposedWaves * kWave * s.c * 4;
                const size_t bytes = x_bytes > sum_bytes ? x_bytes : sum_bytes;
                const T *x_at = static_cast<const T *>(x) + first * ldx;
                auto go = [&](auto kernel) { kernel<<<grid, kTransposedWaves * kWave, bytes, st>>>(a, x_at, ldx, partial, count, s.part); };
                auto by_zeros = [&](auto zeros) {
                    constexpr bool kZero = decltype(zeros)::value;
                    switch (s.m) {
                    case 1: return go(k_q4_mv_t<T, S, kZero, 1, 16, 8>);
                    case 2: return go(k_q4_mv_t<T, S, kZero, 2, 16, 8>);
                    case 4: return go(k_q4_mv_t<T, S, kZero, 4, 8, 4>);
                    case 6: return go(k_q4_mv_t<T, S, kZero, 6, 8, 4>);
                    case 8: return go(k_q4_mv_t<T, S, kZero, 8, 8, 4>);
                    default: return go(k_q4_mv_t<T, S, kZero, 10, 8, 4>);
                    }
                };
                if (a.zeros) by_zeros(std::true_type());
                else by_zeros(std::false_type());
                HBP_HIP(hipGetLastError());
                k_q4_sum_parts<T, S><<<dim3((unsigned)((a.n_cols + kWave - 1) / kWave), (unsigned)((count + 3) / 4)), 256, 0, st>>>(
                    a, x_at, ldx, partial, (int)s.parts, count, static_cast<T *>(y) + first * ldy, ldy);
                HBP_HIP(hipGetLastError());
                first += count;
            }
            return HBP_OK;
        });
    });
}

}  // extern "C"
