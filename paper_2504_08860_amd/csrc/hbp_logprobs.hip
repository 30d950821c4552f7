// Log probabilities of given tokens, entropies and most likely tokens of rows of logits, and the logits' gradient
// (hbp_token_logprobs, hbp_token_logprobs_backward).
#include "hbp_ops.h"

namespace hbp {
namespace {

// The statistics of a part of a row, with m the largest logit in it, s = sum exp(z - m) and u = sum exp(z - m) (z - m), so that
// lse = m + log s and the entropy is log s - u / s.  A part without an unmasked token has m = -inf, s = u = 0.
struct Stats {
    float m, s, u;
};

__device__ __forceinline__ void add_logit(Stats &a, float z)
{
    const float e = __expf(z - a.m);
    a.s += e;
    a.u += e > 0.0f ? e * (z - a.m) : 0.0f;  // (0 times -inf: a masked token, or one too far down to count)
}

__device__ __forceinline__ void move_to(Stats &a, float m)  // m >= a.m
{
    if (m == a.m || !(m > -INFINITY)) return;
    const float d = a.m - m, f = __expf(d);
    a.u = a.s > 0.0f ? f * (a.u + a.s * d) : a.u * f;  // sums from below: (z - m) = (z - a.m) + d
    if (f == 0.0f && a.s == a.s) a.u = 0.0f;
    a.s *= f;
    a.m = m;
}

__device__ __forceinline__ Stats join(Stats a, Stats b)
{
    const float m = fmaxf(a.m, b.m);
    const bool nan = !(a.s == a.s) || !(b.s == b.s);
    move_to(a, m);
    move_to(b, m);
    Stats r{m, a.s + b.s, a.u + b.u};
    if (nan) r.s = NAN;
    return r;
}

__device__ __forceinline__ Stats wave_join(Stats a)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        Stats b{__shfl_xor(a.m, d), __shfl_xor(a.s, d), __shfl_xor(a.u, d)};
        a = join(a, b);
    }
    return a;
}

// A logit and its place as one number that is the larger the earlier it comes among the alternatives: descending value, then
// ascending index.  -0 equals 0, and NaN is the largest.  Below every one of them: 0.
__device__ __forceinline__ uint32_t order_of(float z)
{
    z += 0.0f;
    const uint32_t bits = z == z ? __float_as_uint(z) : 0x7fc00000u;
    return bits ^ ((uint32_t)((int32_t)bits >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint64_t alternative(float z, uint32_t index) { return (uint64_t)order_of(z) << 32 | (uint32_t)~index; }
__device__ __forceinline__ float value_of(uint64_t a)
{
    const uint32_t o = (uint32_t)(a >> 32);
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ int32_t index_of(uint64_t a) { return (int32_t)~(uint32_t)a; }

__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// The `top` (up to 64) first alternatives seen by a wavefront, in order, one to a lane.
struct Best {
    uint64_t mine = 0, last = 0;  // this lane's; the one that a new one has to beat, the same in every lane
    __device__ __forceinline__ void offer(uint64_t a, int top)  // one (or 0) from every lane
    {
        uint64_t waiting = __ballot(a > last);
        while (waiting) {
            const int from = __builtin_ctzll(waiting);
            waiting &= waiting - 1;
            const uint64_t v = lane_value(a, from);
            if (v <= last) continue;
            const int lane = threadIdx.x % kWave;
            const int at = __popcll(__ballot(mine > v));
            const uint64_t above = __shfl_up(mine, 1);
            mine = lane < at ? mine : lane == at ? v : above;
            last = lane_value(mine, top - 1);
        }
    }
};

constexpr int kStatThreads = 512, kStatWaves = kStatThreads / kWave;

struct LogprobArgs {
    const void *logits;
    int64_t ldz, vocabulary, part;  // part: logits of a row that one workgroup takes, a multiple of 8
    const void *ids;
    int32_t id_bytes, top, parts;
    float *logp, *entropy, *lse;
    int32_t *top_ids;
    float *top_logp;
    Stats *stats;        // [tokens][parts]
    uint64_t *best;      // [tokens][parts][top]
};

__device__ __forceinline__ int64_t id_at(const void *ids, int id_bytes, int64_t t)
{
    return id_bytes == 8 ? static_cast<const int64_t *>(ids)[t] : static_cast<const int32_t *>(ids)[t];
}

// what a row's results are, from the statistics and alternatives of all of it; one wavefront
template <typename T> __device__ __forceinline__ void finish_row(const LogprobArgs &p, int64_t t, Stats a, const Best &best)
{
    const int lane = threadIdx.x % kWave;
    const bool none = !(a.m > -INFINITY) && a.s == a.s;  // nothing is left
    const float log_s = logf(a.s);
    // (a.m + log_s would round away what log_s adds to a large m: differences to m are taken first)
    const float lse = none ? -INFINITY : a.m + log_s;
    if (lane == 0) {
        if (p.lse) p.lse[t] = lse;
        if (p.entropy) p.entropy[t] = none ? 0.0f : log_s - a.u / a.s;
        if (p.logp && p.ids) {
            const int64_t id = id_at(p.ids, p.id_bytes, t);
            float v = 0.0f;
            if (id >= p.vocabulary) v = NAN;
            else if (id >= 0) v = none ? -INFINITY : to_f32(static_cast<const T *>(p.logits)[t * p.ldz + id]) - a.m - log_s;
            p.logp[t] = v;
        }
    }
    if (lane < p.top) {
        p.top_ids[t * p.top + lane] = index_of(best.mine);
        p.top_logp[t * p.top + lane] = none ? -INFINITY : value_of(best.mine) - a.m - log_s;
    }
}

template <typename T, bool TOP> __global__ __launch_bounds__(kStatThreads) void k_logprobs(LogprobArgs p)
{
    __shared__ Stats wave_stats[kStatWaves];
    __shared__ uint64_t wave_best[kStatWaves][TOP ? kWave : 1];
    const int64_t t = blockIdx.y;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const T *z = static_cast<const T *>(p.logits) + t * p.ldz;
    const int64_t begin = (int64_t)blockIdx.x * p.part, end = min(begin + p.part, p.vocabulary);
    Stats a{-INFINITY, 0.0f, 0.0f};
    Best best;
    for (int64_t at = begin; at < end; at += kStatThreads * 8) {  // (the same number of turns in every lane: alternatives go by wavefronts)
        const int64_t col = at + threadIdx.x * 8;
        const int64_t left = end - col;
        Eight<T> v;
        if (left > 0) v.load_first(z + col, left);
        if (left > 0) {
            float m = a.m;
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (i < left) m = fmaxf(m, v.get(i));
            move_to(a, m);
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (i < left && (m > -INFINITY || v.get(i) != v.get(i))) add_logit(a, v.get(i));
        }
        if constexpr (TOP)
#pragma unroll
            for (int i = 0; i < 8; i++) best.offer(i < left ? alternative(v.get(i), (uint32_t)(col + i)) : 0, p.top);
    }
    a = wave_join(a);
    if (lane == 0) wave_stats[wave] = a;
    if constexpr (TOP) wave_best[wave][lane] = best.mine;
    __syncthreads();
    if (wave != 0) return;
    a = lane < kStatWaves ? wave_stats[lane] : Stats{-INFINITY, 0.0f, 0.0f};
    a = wave_join(a);
    if constexpr (TOP)
        for (int w = 1; w < kStatWaves; w++) best.offer(lane < p.top ? wave_best[w][lane] : 0, p.top);
    if (p.parts == 1) {
        finish_row<T>(p, t, a, best);
    } else {
        const int64_t at = t * p.parts + blockIdx.x;
        if (lane == 0) p.stats[at] = a;
        if (lane < p.top) p.best[at * p.top + lane] = best.mine;
    }
}

// joins the parts of a row
template <typename T> __global__ __launch_bounds__(kWave) void k_logprobs_join(LogprobArgs p)
{
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x;
    Stats a{-INFINITY, 0.0f, 0.0f};
    for (int i = lane; i < p.parts; i += kWave) a = join(a, p.stats[t * p.parts + i]);
    a = wave_join(a);
    Best best;
    const uint64_t *all = p.best + t * p.parts * p.top;
    const int count = p.parts * p.top;
    for (int i = 0; i < count; i += kWave) best.offer(i + lane < count ? all[i + lane] : 0, p.top);
    finish_row<T>(p, t, a, best);
}

struct LogprobBackArgs {
    const void *logits;
    int64_t ldz, ldd, vocabulary;
    const void *ids;
    int32_t id_bytes;
    const float *lse, *entropy, *g_logp, *g_entropy;
    void *d_logits;
};

template <typename T> __global__ __launch_bounds__(256) void k_logprobs_backward(LogprobBackArgs p)
{
    const int64_t t = blockIdx.y;
    const T *z = static_cast<const T *>(p.logits) + t * p.ldz;
    T *d = static_cast<T *>(p.d_logits) + t * p.ldd;
    const int64_t id = p.ids ? id_at(p.ids, p.id_bytes, t) : -1;
    const float lse = p.lse[t], entropy = p.g_entropy ? p.entropy[t] : 0.0f, w = p.g_entropy ? p.g_entropy[t] : 0.0f;
    float u = id >= 0 && p.g_logp ? p.g_logp[t] : 0.0f;
    if (id >= p.vocabulary && p.g_logp) u = NAN;
    const bool none = lse == -INFINITY;
    const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    const int64_t left = p.vocabulary - col;
    if (left <= 0) return;
    Eight<T> v, out;
    v.load_first(z + col, left);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float lp = v.get(i) - lse;
        const float prob = __expf(lp);
        float g = prob * (u + (prob > 0.0f ? w * (lp + entropy) : 0.0f));
        g = col + i == id ? u - g : -g;
        if (none) g = u == u ? 0.0f : u;
        out.set(i, g);
    }
    out.store_first(d + col, left);
}

// parts of a row: enough workgroups for the chip, none of fewer than 4096 logits
int64_t parts_of(int64_t tokens, int64_t vocabulary)
{
    const int64_t most = (vocabulary + 4095) / 4096, wanted = (512 + tokens - 1) / (tokens > 0 ? tokens : 1);
    const int64_t parts = wanted < most ? wanted : most;
    return parts < 64 ? parts : 64;
}

int check_logits(int type, int64_t ldz, int64_t tokens, int64_t vocabulary)
{
    if (!is_type(type) || tokens < 0 || vocabulary < 1 || (tokens > 1 && ldz < vocabulary)) return HBP_ERR_INVALID_ARGUMENT;
    if (vocabulary > (int64_t(1) << 31) - 512 || tokens > (int64_t(1) << 31) - 512) return HBP_ERR_TOO_LARGE;
    return HBP_OK;
}

}  // namespace
}  // namespace hbp

extern "C" {

int hbp_token_logprobs_workspace(int type, int64_t tokens, int64_t vocabulary, int top, size_t *bytes)
{
    using namespace hbp;
    const int rc = check_logits(type, vocabulary, tokens, vocabulary);
    if (rc != HBP_OK) return rc;
    if (!bytes || top < 0 || top > kWave || top > vocabulary) return HBP_ERR_INVALID_ARGUMENT;
    const int64_t parts = parts_of(tokens, vocabulary);
    *bytes = parts > 1 ? (size_t)(tokens * parts) * (8 * (size_t)top + sizeof(Stats)) : 0;
    return HBP_OK;
}

int hbp_token_logprobs(int type, const void *logits, int64_t ldz, int64_t tokens, int64_t vocabulary, const void *ids, int id_bytes, float *logp,
                       float *entropy, float *lse, int top, int32_t *top_ids, float *top_logp, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace hbp;
    size_t need = 0;
    int rc = hbp_token_logprobs_workspace(type, tokens, vocabulary, top, &need);
    if (rc == HBP_OK) rc = check_logits(type, ldz, tokens, vocabulary);
    if (rc != HBP_OK) return rc;
    if (tokens == 0) return HBP_OK;
    if (!logits || !aligned(logits, type_bytes(type)) || (ids && id_bytes != 4 && id_bytes != 8) || (ids && !aligned(ids, id_bytes))) return HBP_ERR_INVALID_ARGUMENT;
    if ((logp && !ids) || (top > 0 && (!top_ids || !top_logp))) return HBP_ERR_INVALID_ARGUMENT;
    for (const void *p : {(const void *)logp, (const void *)entropy, (const void *)lse, (const void *)top_ids, (const void *)top_logp})
        if (!aligned(p, 4)) return HBP_ERR_INVALID_ARGUMENT;
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return HBP_ERR_INVALID_ARGUMENT;
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    LogprobArgs p{};
    p.logits = logits; p.ldz = ldz; p.vocabulary = vocabulary;
    p.ids = ids; p.id_bytes = id_bytes; p.top = top;
    p.parts = (int32_t)parts_of(tokens, vocabulary);
    p.part = ((vocabulary + p.parts - 1) / p.parts + 7) / 8 * 8;
    p.logp = logp; p.entropy = entropy; p.lse = lse; p.top_ids = top_ids; p.top_logp = top_logp;
    p.best = static_cast<uint64_t *>(workspace);
    p.stats = reinterpret_cast<Stats *>(static_cast<uint64_t *>(workspace) + (p.parts > 1 ? tokens * p.parts * top : 0));
    hipStream_t st = (hipStream_t)stream;
    constexpr int64_t kRows = 32768;  // rows of one launch: the grid's second dimension ends at 65535
    return by_type(type, [&](auto t) -> int {
        using T = decltype(t);
        for (int64_t at = 0; at < tokens; at += kRows) {
            LogprobArgs q = p;
            const int64_t rows = tokens - at < kRows ? tokens - at : kRows;
            q.logits = static_cast<const T *>(logits) + at * ldz;
            q.ids = ids ? static_cast<const char *>(ids) + at * id_bytes : nullptr;
            if (q.logp) q.logp += at;
            if (q.entropy) q.entropy += at;
            if (q.lse) q.lse += at;
            if (top) { q.top_ids += at * top; q.top_logp += at * top; }
            if (p.parts > 1) { q.best += at * p.parts * top; q.stats += at * p.parts; }
            const dim3 grid((unsigned)p.parts, (unsigned)rows);
            if (top) k_logprobs<T, true><<<grid, kStatThreads, 0, st>>>(q);
            else k_logprobs<T, false><<<grid, kStatThreads, 0, st>>>(q);
            HBP_HIP(hipGetLastError());
            if (p.parts > 1) {
                k_logprobs_join<T><<<dim3((unsigned)rows), kWave, 0, st>>>(q);
                HBP_HIP(hipGetLastError());
            }
        }
        return HBP_OK;
    });
}

int hbp_token_logprobs_backward(int type, const void *logits, int64_t ldz, int64_t tokens, int64_t vocabulary, const void *ids, int id_bytes,
                                const float *lse, const float *entropy, const float *g_logp, const float *g_entropy, void *d_logits, int64_t ldd,
                                void *stream)
{
    using namespace hbp;
    int rc = check_logits(type, ldz, tokens, vocabulary);
    if (rc == HBP_OK) rc = check_logits(type, ldd, tokens, vocabulary);
    if (rc != HBP_OK) return rc;
    if (tokens == 0) return HBP_OK;
    if (!logits || !d_logits || !lse || !aligned(logits, type_bytes(type)) || !aligned(d_logits, type_bytes(type))) return HBP_ERR_INVALID_ARGUMENT;
    if ((ids && id_bytes != 4 && id_bytes != 8) || (ids && !aligned(ids, id_bytes)) || (g_logp && !ids) || (g_entropy && !entropy)) return HBP_ERR_INVALID_ARGUMENT;
    for (const float *p : {lse, entropy, g_logp, g_entropy})
        if (!aligned(p, 4)) return HBP_ERR_INVALID_ARGUMENT;
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    constexpr int64_t kRows = 32768;
    return by_type(type, [&](auto t) -> int {
        using T = decltype(t);
        for (int64_t at = 0; at < tokens; at += kRows) {
            const int64_t rows = tokens - at < kRows ? tokens - at : kRows;
            LogprobBackArgs p{};
            p.logits = static_cast<const T *>(logits) + at * ldz; p.ldz = ldz; p.ldd = ldd; p.vocabulary = vocabulary;
            p.ids = ids ? static_cast<const char *>(ids) + at * id_bytes : nullptr; p.id_bytes = id_bytes;
            p.lse = lse + at; p.entropy = entropy ? entropy + at : nullptr;
            p.g_logp = g_logp ? g_logp + at : nullptr; p.g_entropy = g_entropy ? g_entropy + at : nullptr;
            p.d_logits = static_cast<T *>(d_logits) + at * ldd;
            k_logprobs_backward<T><<<dim3((unsigned)((vocabulary + 2047) / 2048), (unsigned)rows), 256, 0, (hipStream_t)stream>>>(p);
            HBP_HIP(hipGetLastError());
        }
        return HBP_OK;
    });
}

}  // extern "C"
