// Residual sum, gate and norms between two blocks, and their gradients (hbp_residual_norms, hbp_residual_norms_backward).
#include "hbp_ops.h"

#include <algorithm>

namespace hbp {
namespace {

constexpr int64_t kMaxWidth = 16384;
constexpr int64_t kMostWorkgroups = int64_t(1) << 21;  // of one forward launch: a grid counts its threads, up to 1024 of each, in 32 bits

struct NormArgs {
    int64_t tokens, ldh, ldy, ldho, ldxo, ldg;
    int32_t width;
    float scale, eps;
    const void *h, *y, *w_post, *w_pre, *gate;
    void *h_out, *x_out;
    float *rstd;
};

// Forward.  A row is a workgroup's or, up to 256 columns, that of 8 to 32 lanes of a one-wavefront workgroup (with 64 lanes for every row, most of them without columns,
// 100000 x 128 with gradients took 144 us, so 80): THREADS threads with CHUNKS times eight columns each, which stay in registers from the only
// read to the writes; two sums over the row lie between.  Bound: HBM; 8192 x 4096 bf16 with a gate for each value 63 us, 5.3 TB/s; one row of 4096 2.6 us.
template <typename T, int THREADS, int CHUNKS, int GATE>
__global__ __launch_bounds__(THREADS < kWave ? kWave : THREADS) void k_residual_norms(NormArgs n)
{
    __shared__ float slots[2][THREADS < kWave ? 1 : THREADS / kWave];
    constexpr int kAtOnce = THREADS < kWave ? kWave / THREADS : 1;  // rows of a workgroup
    const int thread = threadIdx.x % THREADS;
    const int64_t mine = (int64_t)blockIdx.x * kAtOnce + threadIdx.x / THREADS, t = min(mine, n.tokens - 1);  // (behind the last row it is read again)
    const T *h = static_cast<const T *>(n.h) + t * n.ldh, *y = static_cast<const T *>(n.y) + t * n.ldy;
    const T *g = GATE == HBP_GATE_FULL ? static_cast<const T *>(n.gate) + t * n.ldg : static_cast<const T *>(n.gate);
    const T *w_post = static_cast<const T *>(n.w_post), *w_pre = static_cast<const T *>(n.w_pre);
    Eight<T> yy[CHUNKS], hh[CHUNKS], gg[CHUNKS];
    float row_gate = n.scale;
    if constexpr (GATE == HBP_GATE_TOKEN) row_gate *= to_f32(g[t]);
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) {
        const int col = (c * THREADS + thread) * 8;
        yy[c].load_first(y + col, n.width - col);
        hh[c].load_first(h + col, n.width - col);
        if constexpr (GATE == HBP_GATE_FULL || GATE == HBP_GATE_CHANNEL) gg[c].load_first(g + col, n.width - col);
    }
    float sum[1] = {0};
#pragma unroll
    for (int c = 0; c < CHUNKS; c++)
#pragma unroll
        for (int i = 0; i < 8; i++) sum[0] += yy[c].get(i) * yy[c].get(i);
    block_sums<1, THREADS>(sum, slots[0]);
    const float r1 = rsqrtf(sum[0] / n.width + n.eps);
    float next[CHUNKS][8];
    sum[0] = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) {
        const int col = (c * THREADS + thread) * 8;
        Eight<T> w;
        if (w_post) w.load_first(w_post + col, n.width - col);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            float v = yy[c].get(i) * r1;
            if (w_post) v *= w.get(i);
            if constexpr (GATE == HBP_GATE_FULL || GATE == HBP_GATE_CHANNEL) v *= gg[c].get(i);
            next[c][i] = hh[c].get(i) + row_gate * v;
            sum[0] += next[c][i] * next[c][i];
        }
    }
    block_sums<1, THREADS>(sum, slots[1]);
    const float r2 = rsqrtf(sum[0] / n.width + n.eps);
    if (mine != t) return;
    T *h_out = static_cast<T *>(n.h_out) + t * n.ldho, *x_out = static_cast<T *>(n.x_out) + t * n.ldxo;
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) {
        const int col = (c * THREADS + thread) * 8;
        Eight<T> w, a, b;
        if (w_pre) w.load_first(w_pre + col, n.width - col);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            a.set(i, next[c][i]);
            const float v = next[c][i] * r2;
            b.set(i, w_pre ? v * w.get(i) : v);
        }
        a.store_first(h_out + col, n.width - col);
        b.store_first(x_out + col, n.width - col);
    }
    if (n.rstd && thread == 0) {
        n.rstd[2 * t] = r1;
        n.rstd[2 * t + 1] = r2;
    }
}

struct NormBackArgs {
    int64_t tokens, ldh, ldy, ldg, lddho, lddxo, lddh, lddy;
    int32_t width;
    float scale;
    const void *d_h_out, *d_x_out, *h, *y, *w_post, *w_pre, *gate;
    const float *rstd;
    void *d_h, *d_y, *d_gate;
    float *partial;  // [workgroups times rows at once][3][width]: d_w_post, d_w_pre, a CHANNEL's d_gate
};

// Two sums of each of a thread's columns: in registers or, where a thread has 32 columns and their rows leave no registers for them, in LDS, each thread's own.
template <int THREADS, int CHUNKS> struct Sums {
    static constexpr bool kInLds = CHUNKS > 2;
    static constexpr size_t kBytes = kInLds ? sizeof(float) * 2 * CHUNKS * 8 * THREADS : 0;
    float v[2][kInLds ? 1 : CHUNKS][8];
    int thread;
    static __device__ __forceinline__ float4 *lds()
    {
        extern __shared__ float4 sums_in_lds[];
        return sums_in_lds;
    }
    __device__ __forceinline__ float4 &place(int which, int c, int half) const { return lds()[((which * CHUNKS + c) * 2 + half) * THREADS + thread]; }
    __device__ __forceinline__ Sums(int t) : v{}, thread(t)
    {
        if constexpr (kInLds)
#pragma unroll
            for (int i = 0; i < 4 * CHUNKS; i++) lds()[i * THREADS + thread] = float4{0, 0, 0, 0};
    }
    __device__ __forceinline__ void add(int which, int c, const float (&x)[8])
    {
        if constexpr (kInLds) {
#pragma unroll
            for (int half = 0; half < 2; half++) {
                float4 &s = place(which, c, half);
                s = float4{s.x + x[4 * half], s.y + x[4 * half + 1], s.z + x[4 * half + 2], s.w + x[4 * half + 3]};
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) v[which][c][i] += x[i];
        }
    }
    __device__ __forceinline__ void get(int which, int c, float (&x)[8]) const
    {
        if constexpr (kInLds) {
#pragma unroll
            for (int half = 0; half < 2; half++) {
                const float4 s = place(which, c, half);
                x[4 * half] = s.x; x[4 * half + 1] = s.y; x[4 * half + 2] = s.z; x[4 * half + 3] = s.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = v[which][c][i];
        }
    }
};

// Backward.  With the normed rows u = r1 y and v = r2 h' and a = d_x_out w_pre, e = d_h_out + r2 (a - v mean(a v)) is d_h, and b = scale g w_post e goes through the
// first norm: d_y = r1 (b - u mean(b u)).  e in the second mean is spelled out, so that all three sums of a row, of
// a v, of w u (d_h_out + r2 a) and of w u v with w = scale g w_post, are taken together: one wait for the others per row.  The sums are over normed rows, so that no
// power of r1 or r2 is formed, which may be no fp32 number.
// h' is computed again from h, y and the gate, which are read anyway: not the rounded one, and no read more.
//
// A workgroup walks through every so many rows and keeps its columns' sums for the weights; workgroups' sums are added by a second kernel, in their
// order.  Of a row, what was read stays in registers as it came (h' is cheaper to compute twice than to keep), and so do, up to 16 columns a thread, the weights.  512 threads at
// most: with 1024 a row of 16384 columns does not fit their 128 registers.  With 512 it fits their 256 if nothing else is kept there: the sums are in LDS, 128 KB, the weights are read again for each
// row, from the caches, and the compiler is not to keep what it made of a row from one walk through it to the next.  2048 x 16384 fp32 with a gate for each column 283 us, with all of it in
// registers, of which 661 were spilled, 606 (still spilled: 19 of fp32 rows with such a gate, 12 with one for each value).
// Bound: HBM; 8192 x 4096 bf16 with a gate for each value 113 us, 4.7 TB/s, and 5 for the workgroups' sums (39 with four shares and one load at a time).
template <typename T, int THREADS, int CHUNKS, int GATE>
__global__ __launch_bounds__(THREADS < kWave ? kWave : THREADS) void k_residual_norms_backward(NormBackArgs n)
{
    __shared__ float slots[2][THREADS < kWave ? 1 : THREADS / kWave * 3];
    constexpr int kAtOnce = THREADS < kWave ? kWave / THREADS : 1;  // rows of a workgroup
    const int thread = threadIdx.x % THREADS, of_these = threadIdx.x / THREADS;
    constexpr bool kFull = GATE == HBP_GATE_FULL, kChannel = GATE == HBP_GATE_CHANNEL;
    constexpr bool kKeep = !Sums<THREADS, CHUNKS>::kInLds;  // the weights
    constexpr int kWeights = kKeep ? CHUNKS : 1;
    Eight<T> wp[kWeights], wq[kWeights], gg[kFull ? CHUNKS : kWeights];
    auto load_weights = [&](int c, int to) {
        const int col = (c * THREADS + thread) * 8, left = n.width - col;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            wp[to].set(i, 1.0f);
            wq[to].set(i, 1.0f);
        }
        if (n.w_post) wp[to].load_first(static_cast<const T *>(n.w_post) + col, left);
        if (n.w_pre) wq[to].load_first(static_cast<const T *>(n.w_pre) + col, left);
        if constexpr (kChannel) gg[to].load_first(static_cast<const T *>(n.gate) + col, left);
    };
    if constexpr (kKeep)
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) load_weights(c, c);
    Sums<THREADS, CHUNKS> sums(thread);
    const float inverse_width = 1.0f / n.width;
    int odd = 0;
    for (int64_t t0 = (int64_t)blockIdx.x * kAtOnce; t0 < n.tokens; t0 += (int64_t)gridDim.x * kAtOnce, odd ^= 1) {
        const bool mine = t0 + of_these < n.tokens;  // (behind the last row it is read again, for nothing)
        const int64_t t = mine ? t0 + of_these : n.tokens - 1;
        const T *h = static_cast<const T *>(n.h) + t * n.ldh, *y = static_cast<const T *>(n.y) + t * n.ldy;
        const float r1 = n.rstd[2 * t], r2 = n.rstd[2 * t + 1];
        const float row_gate = GATE == HBP_GATE_TOKEN ? to_f32(static_cast<const T *>(n.gate)[t]) : 1.0f;
        Eight<T> yy[CHUNKS], hh[CHUNKS], dx[CHUNKS], dh[CHUNKS];
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int col = (c * THREADS + thread) * 8, left = n.width - col;
            yy[c].load_first(y + col, left);
            hh[c].load_first(h + col, left);
            dx[c].clear();
            dh[c].clear();
            if (n.d_x_out) dx[c].load_first(static_cast<const T *>(n.d_x_out) + t * n.lddxo + col, left);
            if (n.d_h_out) dh[c].load_first(static_cast<const T *>(n.d_h_out) + t * n.lddho + col, left);
            if constexpr (kFull) gg[c].load_first(static_cast<const T *>(n.gate) + t * n.ldg + col, left);
        }
        float sum[3] = {0, 0, 0};
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int k = kKeep ? c : 0, kg = kKeep || kFull ? c : 0;
            if constexpr (!kKeep) load_weights(c, 0);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                float w = n.scale * wp[k].get(i);
                if constexpr (kFull || kChannel) w *= gg[kg].get(i);
                const float wu = w * (yy[c].get(i) * r1), hat = (hh[c].get(i) + row_gate * wu) * r2, a = dx[c].get(i) * wq[k].get(i);
                sum[0] += a * hat;
                sum[1] += wu * (dh[c].get(i) + r2 * a);
                sum[2] += wu * hat;
            }
        }
        block_sums<3, THREADS>(sum, slots[odd]);
        if (!mine) continue;
        if constexpr (!kKeep)
#pragma unroll
            for (int c = 0; c < CHUNKS; c++) {
                yy[c].forget();
                hh[c].forget();
                dx[c].forget();
            }
        const float along2 = r2 * (sum[0] * inverse_width);
        const float through = sum[1] - along2 * sum[2];  // sum of b u, a row's gate left out
        const float along1 = row_gate * through * inverse_width;
        if (GATE == HBP_GATE_TOKEN && n.d_gate && thread == 0) static_cast<float *>(n.d_gate)[t] = through;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int col = (c * THREADS + thread) * 8, left = n.width - col;
            Eight<T> de, dy, dg;
            float post[8], pre[8];
            const int k = kKeep ? c : 0, kg = kKeep || kFull ? c : 0;
            if constexpr (!kKeep) load_weights(c, 0);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float yv = yy[c].get(i), xv = dx[c].get(i), w_post = wp[k].get(i);
                float gate = n.scale * row_gate;
                if constexpr (kFull || kChannel) gate *= gg[kg].get(i);
                const float unit = yv * r1, hat = (hh[c].get(i) + gate * (unit * w_post)) * r2;
                const float e = dh[c].get(i) + r2 * (xv * wq[k].get(i)) - along2 * hat;
                de.set(i, e);
                dy.set(i, r1 * (gate * e * w_post - along1 * unit));
                post[i] = (kChannel ? n.scale : gate) * e * unit;
                pre[i] = xv * hat;
                if constexpr (kFull) dg.set(i, n.scale * e * (unit * w_post));
            }
            sums.add(0, c, post);
            sums.add(1, c, pre);
            de.store_first(static_cast<T *>(n.d_h) + t * n.lddh + col, left);
            dy.store_first(static_cast<T *>(n.d_y) + t * n.lddy + col, left);
            if constexpr (kFull)
                if (n.d_gate) dg.store_first(static_cast<T *>(n.d_gate) + t * n.ldg + col, left);
        }
    }
    float *partial = n.partial + ((int64_t)blockIdx.x * kAtOnce + of_these) * 3 * n.width;
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) {
        const int col = (c * THREADS + thread) * 8;
        float post[8], pre[8];
        sums.get(0, c, post);
        sums.get(1, c, pre);
        const int k = kKeep ? c : 0;
        if constexpr (kChannel && !kKeep) load_weights(c, 0);
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (col + i < n.width) {  // (a CHANNEL's gate and w_post are the same in every row: one sum for both)
                partial[col + i] = kChannel ? gg[k].get(i) * post[i] : post[i];
                partial[n.width + col + i] = pre[i];
                if constexpr (kChannel) partial[2 * n.width + col + i] = wp[k].get(i) * post[i];
            }
    }
}

// out[which][col] = sum over the workgroups of partial[workgroup][which][col]: sixteen shares of them, each in ascending order, then the shares
constexpr int kShares = 16;
__global__ __launch_bounds__(kShares * 64) void k_norm_weight_sums(const float *partial, int32_t workgroups, int32_t width, float *d_w_post, float *d_w_pre, float *d_gate)
{
    __shared__ float shares[kShares][64];
    const int lane = threadIdx.x % 64, share = threadIdx.x / 64, col = blockIdx.x * 64 + lane;
    float *out = blockIdx.y == 0 ? d_w_post : blockIdx.y == 1 ? d_w_pre : d_gate;
    if (!out) return;
    float sum = 0;
    if (col < width) {
        const float *at = partial + (int64_t)blockIdx.y * width + col;
        const int64_t apart = 3 * (int64_t)width;
        int b = share;
        for (; b + 7 * kShares < workgroups; b += 8 * kShares) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; k++) v[k] = at[(b + k * kShares) * apart];
#pragma unroll
            for (int k = 0; k < 8; k++) sum += v[k];
        }
        for (; b < workgroups; b += kShares) sum += at[b * apart];
    }
    shares[share][lane] = sum;
    __syncthreads();
    if (share == 0 && col < width) {
        sum = 0;
        for (int k = 0; k < kShares; k++) sum += shares[k][lane];
        out[col] = sum;
    }
}

// Threads and chunks for a width: f(threads, chunks) as compile-time constants
template <int V> struct Int { static constexpr int value = V; };
template <typename F> int by_width_forward(int64_t width, F f)
{
    if (width <= 64) return f(Int<8>(), Int<1>());
    if (width <= 128) return f(Int<16>(), Int<1>());
    if (width <= 256) return f(Int<32>(), Int<1>());
    if (width <= 512) return f(Int<64>(), Int<1>());
    if (width <= 2048) return f(Int<256>(), Int<1>());
    if (width <= 4096) return f(Int<512>(), Int<1>());
    if (width <= 8192) return f(Int<1024>(), Int<1>());
    return f(Int<1024>(), Int<2>());
}
template <typename F> int by_width_backward(int64_t width, F f)
{
    if (width <= 64) return f(Int<8>(), Int<1>());
    if (width <= 128) return f(Int<16>(), Int<1>());
    if (width <= 256) return f(Int<32>(), Int<1>());
    if (width <= 512) return f(Int<64>(), Int<1>());
    if (width <= 1024) return f(Int<128>(), Int<1>());
    if (width <= 2048) return f(Int<256>(), Int<1>());
    if (width <= 4096) return f(Int<512>(), Int<1>());
    if (width <= 8192) return f(Int<512>(), Int<2>());
    return f(Int<512>(), Int<4>());
}
template <typename F> int by_gate(int kind, F f)
{
    switch (kind) {
    case HBP_GATE_NONE: return f(Int<HBP_GATE_NONE>());
    case HBP_GATE_CHANNEL: return f(Int<HBP_GATE_CHANNEL>());
    case HBP_GATE_TOKEN: return f(Int<HBP_GATE_TOKEN>());
    default: return f(Int<HBP_GATE_FULL>());
    }
}

int64_t rows_at_once(int64_t width) { return width <= 64 ? 8 : width <= 128 ? 4 : width <= 256 ? 2 : 1; }  // of a workgroup

// as many as are on the chip at once: 16 wavefronts for each of 256 compute units, with sums in LDS 8; no more than there are rows, and of narrow rows four turns each
int64_t backward_workgroups(int64_t tokens, int64_t width)
{
    const int64_t threads = width <= 512 ? 64 : width <= 1024 ? 128 : width <= 2048 ? 256 : 512, at_once = rows_at_once(width);
    const int64_t most = width > 8192 ? 256 : 256 * 1024 / threads / at_once, turns = (tokens + at_once - 1) / at_once, enough = threads < 512 ? (turns + 3) / 4 : turns;
    return enough < most ? enough : most;
}

int check_norms(const hbp_norms_t *n)
{
    if (!n || n->tokens < 0 || n->width < 1 || !is_type(n->type) || n->gate_kind < HBP_GATE_NONE || n->gate_kind > HBP_GATE_FULL) return HBP_ERR_INVALID_ARGUMENT;
    if ((n->gate != nullptr) != (n->gate_kind != HBP_GATE_NONE) && n->tokens > 0) return HBP_ERR_INVALID_ARGUMENT;
    if (n->gate_kind == HBP_GATE_FULL && n->ldg < n->width) return HBP_ERR_INVALID_ARGUMENT;
    if (!(n->eps > 0)) return HBP_ERR_INVALID_ARGUMENT;
    const int64_t bytes = type_bytes(n->type);
    if (!aligned(n->w_post, bytes) || !aligned(n->w_pre, bytes) || !aligned(n->gate, bytes)) return HBP_ERR_INVALID_ARGUMENT;
    if (n->width > kMaxWidth || n->tokens >= (int64_t(1) << 31)) return HBP_ERR_TOO_LARGE;
    return HBP_OK;
}

}  // namespace
}  // namespace hbp

extern "C" {

int hbp_residual_norms(const hbp_norms_t *n, const void *h, int64_t ldh, const void *y, int64_t ldy, void *h_out, int64_t ldho, void *x_out,
                       int64_t ldxo, float *rstd, void *stream)
{
    using namespace hbp;
    int rc = check_norms(n);
    if (rc != HBP_OK) return rc;
    if (n->tokens == 0) return HBP_OK;
    const int64_t bytes = type_bytes(n->type);
    for (const void *p : {h, y, (const void *)h_out, (const void *)x_out})
        if (!p || !aligned(p, bytes)) return HBP_ERR_INVALID_ARGUMENT;
    for (int64_t ld : {ldh, ldy, ldho, ldxo})
        if (ld < n->width) return HBP_ERR_INVALID_ARGUMENT;
    if (!aligned(rstd, 4)) return HBP_ERR_INVALID_ARGUMENT;
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    NormArgs a{};
    a.tokens = n->tokens; a.width = (int32_t)n->width;
    a.ldh = ldh; a.ldy = ldy; a.ldho = ldho; a.ldxo = ldxo; a.ldg = n->ldg;
    a.scale = n->scale; a.eps = n->eps;
    a.h = h; a.y = y; a.w_post = n->w_post; a.w_pre = n->w_pre; a.gate = n->gate;
    a.h_out = h_out; a.x_out = x_out; a.rstd = rstd;
    return by_type(n->type, [&](auto type) -> int {
        using T = decltype(type);
        return by_gate(n->gate_kind, [&](auto gate) -> int {
            return by_width_forward(n->width, [&](auto threads, auto chunks) -> int {
                constexpr int kThreads = decltype(threads)::value;
                const int64_t at_once = rows_at_once(n->width);
                for (int64_t first = 0; first < n->tokens; first += kMostWorkgroups * at_once) {
                    NormArgs q = a;
                    q.tokens = std::min(n->tokens - first, kMostWorkgroups * at_once);
                    q.h = static_cast<const T *>(h) + first * ldh;
                    q.y = static_cast<const T *>(y) + first * ldy;
                    q.h_out = static_cast<T *>(h_out) + first * ldho;
                    q.x_out = static_cast<T *>(x_out) + first * ldxo;
                    if (n->gate_kind == HBP_GATE_TOKEN) q.gate = static_cast<const T *>(n->gate) + first;
                    if (n->gate_kind == HBP_GATE_FULL) q.gate = static_cast<const T *>(n->gate) + first * n->ldg;
                    if (rstd) q.rstd = rstd + 2 * first;
                    k_residual_norms<T, kThreads, decltype(chunks)::value, decltype(gate)::value>
                        <<<dim3((unsigned)((q.tokens + at_once - 1) / at_once)), std::max(kThreads, kWave), 0, (hipStream_t)stream>>>(q);
                    HBP_HIP(hipGetLastError());
                }
                return HBP_OK;
            });
        });
    });
}

int hbp_residual_norms_backward_workspace(const hbp_norms_t *n, size_t *bytes)
{
    const int rc = hbp::check_norms(n);
    if (rc != HBP_OK || !bytes) return rc != HBP_OK ? rc : HBP_ERR_INVALID_ARGUMENT;
    *bytes = (size_t)(hbp::backward_workgroups(n->tokens, n->width) * hbp::rows_at_once(n->width) * 3 * n->width) * sizeof(float);
    return HBP_OK;
}

int hbp_residual_norms_backward(const hbp_norms_t *n, const void *d_h_out, int64_t lddho, const void *d_x_out, int64_t lddxo, const void *h,
                                int64_t ldh, const void *y, int64_t ldy, const float *rstd, void *d_h, int64_t lddh, void *d_y, int64_t lddy,
                                float *d_w_post, float *d_w_pre, void *d_gate, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace hbp;
    size_t need = 0;
    int rc = hbp_residual_norms_backward_workspace(n, &need);
    if (rc != HBP_OK) return rc;
    const int64_t bytes = type_bytes(n->type);
    if (n->tokens > 0) {
        for (const void *p : {h, y, (const void *)rstd, (const void *)d_h, (const void *)d_y})
            if (!p || !aligned(p, bytes)) return HBP_ERR_INVALID_ARGUMENT;
        for (int64_t ld : {ldh, ldy, lddh, lddy, d_h_out ? lddho : n->width, d_x_out ? lddxo : n->width})
            if (ld < n->width) return HBP_ERR_INVALID_ARGUMENT;
        if (!aligned(d_h_out, bytes) || !aligned(d_x_out, bytes)) return HBP_ERR_INVALID_ARGUMENT;
    }
    if (!aligned(rstd, 4) || !aligned(d_w_post, 4) || !aligned(d_w_pre, 4) || !aligned(d_gate, n->gate_kind == HBP_GATE_FULL ? bytes : 4)) return HBP_ERR_INVALID_ARGUMENT;
    if (n->gate_kind == HBP_GATE_NONE && d_gate) return HBP_ERR_INVALID_ARGUMENT;
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return HBP_ERR_INVALID_ARGUMENT;
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    const int32_t workgroups = (int32_t)backward_workgroups(n->tokens, n->width);
    hipStream_t st = (hipStream_t)stream;
    if (workgroups > 0) {
        NormBackArgs a{};
        a.tokens = n->tokens; a.width = (int32_t)n->width;
        a.ldh = ldh; a.ldy = ldy; a.ldg = n->ldg; a.lddho = lddho; a.lddxo = lddxo; a.lddh = lddh; a.lddy = lddy;
        a.scale = n->scale;
        a.d_h_out = d_h_out; a.d_x_out = d_x_out; a.h = h; a.y = y; a.w_post = n->w_post; a.w_pre = n->w_pre; a.gate = n->gate;
        a.rstd = rstd; a.d_h = d_h; a.d_y = d_y; a.d_gate = d_gate;
        a.partial = static_cast<float *>(workspace);
        rc = by_type(n->type, [&](auto type) -> int {
            using T = decltype(type);
            return by_gate(n->gate_kind, [&](auto gate) -> int {
                return by_width_backward(n->width, [&](auto threads, auto chunks) -> int {
                    constexpr int kThreads = decltype(threads)::value;
                    constexpr size_t kLds = Sums<kThreads, decltype(chunks)::value>::kBytes;
                    auto kernel = k_residual_norms_backward<T, kThreads, decltype(chunks)::value, decltype(gate)::value>;
                    if (kLds) HBP_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds));
                    kernel<<<dim3((unsigned)workgroups), std::max(kThreads, kWave), kLds, st>>>(a);
                    HBP_HIP(hipGetLastError());
                    return HBP_OK;
                });
            });
        });
        if (rc != HBP_OK) return rc;
    }
    float *channel = n->gate_kind == HBP_GATE_CHANNEL ? static_cast<float *>(d_gate) : nullptr;
    if (d_w_post || d_w_pre || channel) {
        k_norm_weight_sums<<<dim3((unsigned)((n->width + 63) / 64), channel ? 3 : 2), kShares * 64, 0, st>>>(
            static_cast<const float *>(workspace), workgroups * (int32_t)rows_at_once(n->width), (int32_t)n->width, d_w_post, d_w_pre, channel);
        HBP_HIP(hipGetLastError());
    }
    return HBP_OK;
}

}  // extern "C"
