// Log probabilities of given tokens, entropies and most likely tokens of rows of logits, and the logits' gradient
// (hbp_token_logprobs, hbp_token_logprobs_backward).
#include "hbp_ops.h"

namespace hbp {
namespace {

// The statistics of a part of a row, with m the largest logit in it (the lowest number there is: none) and d = (z - m) / log 2: s = sum 2^d and u = sum d 2^d,
// so that lse = m + log s and the entropy is log s - u log 2 / s.  A part without an unmasked token has s = u = 0.
struct Stats {
    float m, s, u;
};
constexpr float kLowest = -3.4028234663852886e38f, kPerLog2 = 1.4426950408889634f, kLog2 = 0.6931471805599453f;
constexpr float kFar = -1000.0f;  // 2 to it is 0; stands for what lies further down, where 0 times it has to be 0

__device__ __forceinline__ void move_to(Stats &a, float m)  // m >= a.m; sums from below: each d grows by the same
{
    const float d = fmaxf((a.m - m) * kPerLog2, kFar), f = __builtin_amdgcn_exp2f(d);
    a.u = f * (a.u + a.s * d);
    a.s *= f;
    a.m = m;
}

// (A NaN makes s NaN: the largest logit passes it over, but its own exponential does not.)
__device__ __forceinline__ void add_eight(Stats &a, const float (&z)[8])
{
    float m = a.m;
#pragma unroll
    for (int i = 0; i < 8; i += 2) asm("v_max3_f32 %0, %1, %2, %0" : "+v"(m) : "v"(z[i]), "v"(z[i + 1]));  // (fmaxf would make each value canonical first)
    if (m > a.m) move_to(a, m);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        // (z / log 2 - m / log 2 would be one instruction, and off by as much as a large m's last bits)
        const float d = (z[i] - m) * kPerLog2, e = __builtin_amdgcn_exp2f(d);
        a.s += e;
        a.u += e * fmaxf(d, kFar);
    }
}

// of all lanes, the same in each: the largest logit first, so that each lane's sums are moved once
__device__ __forceinline__ Stats wave_join(Stats a)
{
    move_to(a, wave_max(a.m));
    return Stats{a.m, wave_sum(a.s), wave_sum(a.u)};
}

// A logit as a number that is the larger the earlier it comes among the alternatives: -0 equals 0, NaN is the largest, and none is 0.  With the complement of
// its index below it, it is an alternative: descending value, then ascending index.
__device__ __forceinline__ uint32_t order_of(float z)
{
    z += 0.0f;
    const uint32_t bits = z == z ? __float_as_uint(z) : 0x7fc00000u;
    return bits ^ ((uint32_t)((int32_t)bits >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint64_t a)
{
    const uint32_t o = (uint32_t)(a >> 32);
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ int32_t index_of(uint64_t a) { return (int32_t)~(uint32_t)a; }

constexpr int kMostThreads = 512, kMostWaves = kMostThreads / kWave, kMostTop = kWave;

struct LogprobArgs {
    const void *logits;
    int64_t ldz, vocabulary, part;  // part: logits of a row that one workgroup takes, a multiple of 8
    const void *ids;
    int32_t id_bytes, top, parts;
    float *logp, *entropy, *lse;
    int32_t *top_ids;
    float *top_logp;
    Stats *stats;        // [tokens][parts]
    uint64_t *best;      // [tokens][parts][top], 0 where there are fewer
};

__device__ __forceinline__ int64_t id_at(const void *ids, int id_bytes, int64_t t)
{
    return id_bytes == 8 ? static_cast<const int64_t *>(ids)[t] : static_cast<const int32_t *>(ids)[t];
}

// The alternatives in question, in LDS: `count` of them in any order, all different.  What is kept of them is the `top` first, found by counting for each
// how many come before it.
template <int MOST> struct Candidates {
    uint64_t all[MOST], sorted[kMostTop];
    int count;
    __device__ __forceinline__ void append(uint64_t a) { all[atomicAdd(&count, 1)] = a; }
    // all threads, behind a barrier; behind the next one `sorted` holds the first ones (as many as there are, up to top)
    __device__ __forceinline__ void select(int top)
    {
        const int n = count;
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const uint64_t a = all[i];
            int before = 0, j = 0;
            for (; j + 8 <= n; j += 8) {
                uint64_t b[8];
#pragma unroll
                for (int k = 0; k < 8; k++) b[k] = all[j + k];
#pragma unroll
                for (int k = 0; k < 8; k++) before += b[k] > a ? 1 : 0;
            }
            for (; j < n; j++) before += all[j] > a ? 1 : 0;
            if (before < top) sorted[before] = a;
        }
    }
};

// The one of the lanes that has `rank` others before it, larger ones and equal ones of lower lanes; 0 where that is none or 0.
__device__ __forceinline__ uint32_t of_rank(uint32_t a, int rank)
{
    int before = 0;
#pragma unroll 8
    for (int j = 0; j < kWave; j++) {
        const uint32_t b = (uint32_t)__builtin_amdgcn_readlane((int)a, j);
        const uint64_t higher = ~0ull << j << 1;  // lanes above j
        before += (__ballot(b > a) | (__ballot(b == a) & higher)) >> (threadIdx.x % kWave) & 1;
    }
    const uint64_t lanes = __ballot(before == rank);
    return lanes ? (uint32_t)__builtin_amdgcn_readlane((int)a, __builtin_ctzll(lanes)) : 0;
}

// what a row's results are, from the statistics and alternatives of all of it
template <typename T> __device__ __forceinline__ void finish_row(const LogprobArgs &p, int64_t t, Stats a, const uint64_t *sorted)
{
    const bool none = a.s == 0.0f;  // nothing is left
    const float log_s = logf(a.s);
    // (a.m + log_s would round away what log_s adds to a large m: differences to m are taken first)
    if (threadIdx.x == 0) {
        if (p.lse) p.lse[t] = none ? -INFINITY : a.m + log_s;
        if (p.entropy) p.entropy[t] = none ? 0.0f : log_s - kLog2 * (a.u / a.s);
        if (p.logp && p.ids) {
            const int64_t id = id_at(p.ids, p.id_bytes, t);
            float v = 0.0f;
            if (id >= p.vocabulary) v = NAN;
            else if (id >= 0) v = none ? -INFINITY : to_f32(static_cast<const T *>(p.logits)[t * p.ldz + id]) - a.m - log_s;
            p.logp[t] = v;
        }
    }
    if ((int)threadIdx.x < p.top) {
        const uint64_t best = sorted[threadIdx.x];
        p.top_ids[t * p.top + threadIdx.x] = index_of(best);
        p.top_logp[t * p.top + threadIdx.x] = none ? -INFINITY : value_of(best) - a.m - log_s;
    }
}

// One pass over a part of a row: statistics in every lane, eight logits at a time.  Bound: HBM; 4096 x 32000 bf16 52 us, 5 TB/s, x 32001 (rows at odd addresses) 64, 79 behind 262 MB of
// writes; some 100 vector instructions, nine of them exponentials, for a wavefront's 512 logits.  Alternatives: barriers and the selection, 8 us for one row in 32 parts,
// 15 for 64 rows of 50001 in 13.
//
// Alternatives: the threads' eights of one turn are a block.  Whatever is below `least` (as order_of has it) cannot be among the top first ones, so only lanes whose largest
// of eight is not matter, and after the first block hardly any is.  In a block with such lanes `least` is raised before anything is handed over: to the top'th of
// the first top / waves lanes' largest of all wavefronts, which for logits in no order leaves about as many candidates as are wanted; and, in a wavefront with more than
// top such lanes all the same, to its own top'th one, so that it hands over no more than 8 top, whatever the order.  Of logits that equal `least` the
// first top lanes' do.
template <typename T, bool TOP, int UNROLL> __global__ __launch_bounds__(kMostThreads) void k_logprobs(LogprobArgs p)
{
    __shared__ Stats wave_stats[kMostWaves];
    __shared__ uint32_t wave_first[TOP ? kWave : 1], block_least;
    __shared__ Candidates<TOP ? 8 * kMostThreads + kMostTop : 1> candidates;  // (a block and what is kept)
    const int64_t t = blockIdx.y;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
    const T *z = static_cast<const T *>(p.logits) + t * p.ldz;
    const int64_t begin = (int64_t)blockIdx.x * p.part, end = min(begin + p.part, p.vocabulary);
    const int block = blockDim.x * 8;
    Stats a{kLowest, 0.0f, 0.0f};
    uint32_t least = 1;
    if constexpr (TOP)
        if (threadIdx.x == 0) candidates.count = 0;
    // (columns count from the part's first one on, in 32 bits)
    const int count = (int)(end - begin), turn = UNROLL * block, last = count - 8;
    const T *part = z + begin;
    const bool few = p.vocabulary < 8;
    auto load = [&](Eight<T> (&v)[UNROLL], int at) {
        if (at + turn <= count) {
#pragma unroll
            for (int k = 0; k < UNROLL; k++) v[k].load(part + at + k * block + threadIdx.x * 8);
        } else if (!few) {  // (the eight that reach beyond the end are read from 8 logits before it: no load depends on a condition)
#pragma unroll
            for (int k = 0; k < UNROLL; k++) v[k].load(part + min(at + k * block + (int)threadIdx.x * 8, last));
        } else {
            v[0].load_first(part, threadIdx.x == 0 ? count : 0);
        }
    };
    auto take = [&](const Eight<T> (&v)[UNROLL], int at) {
#pragma unroll
        for (int k = 0; k < UNROLL; k++) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; i++) f[i] = v[k].get(i);
            const int mine_at = at + k * block + threadIdx.x * 8;
            int col = mine_at, from = 0, to = 8;  // the eight's first column, and which of them are this thread's
            if (at + turn > count) {
                col = few ? 0 : min(mine_at, last);
                from = min(mine_at - col, 8);
                to = min(count - col, 8);
                if (from > 0 || to < 8)
#pragma unroll
                    for (int i = 0; i < 8; i++) f[i] = i >= from && i < to ? f[i] : -INFINITY;
            }
            add_eight(a, f);
            if constexpr (TOP) {
                if (at + k * block >= count) break;  // (the same in every thread)
                float largest = -INFINITY;
                bool nan = false;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    largest = fmaxf(largest, f[i]);
                    nan |= f[i] != f[i];
                }
                const uint32_t first = from < to ? order_of(nan ? NAN : largest) : 0;
                if (!__syncthreads_or(first >= least)) continue;
                const int firsts = min((p.top + waves - 1) / waves, kWave / waves);
                uint32_t left = first >= least ? first : 0;
                for (int i = 0; i < firsts; i++) {
                    const uint32_t largest_left = wave_max(left);
                    if (lane == 0) wave_first[wave * firsts + i] = largest_left;
                    if (lane == __builtin_ctzll(__ballot(left == largest_left))) left = 0;
                }
                __syncthreads();
                if (wave == 0) {
                    const uint32_t raised = of_rank(lane < waves * firsts ? wave_first[lane] : 0, p.top - 1);
                    if (lane == 0) block_least = max(least, raised);
                }
                __syncthreads();
                least = block_least;
                uint32_t mine = least;
                if (__popcll(__ballot(first >= least)) > p.top) mine = max(least, of_rank(first, p.top - 1));
                if (__ballot(first >= mine)) {
                    uint32_t order[8];
                    bool equal = false;
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        order[i] = i >= from && i < to ? order_of(f[i]) : 0;
                        equal |= order[i] == mine;
                    }
                    if (__popcll(__ballot(equal) & ((1ull << lane) - 1)) >= p.top) mine++;
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        if (order[i] >= mine) candidates.append((uint64_t)order[i] << 32 | (uint32_t) ~(uint32_t)(begin + col + i));
                }
                __syncthreads();
                candidates.select(p.top);
                const int n = candidates.count;
                __syncthreads();
                if ((int)threadIdx.x < min(n, p.top)) candidates.all[threadIdx.x] = candidates.sorted[threadIdx.x];
                if (threadIdx.x == 0) candidates.count = min(n, p.top);
                if (n >= p.top) least = (uint32_t)(candidates.sorted[p.top - 1] >> 32) + 1;  // (an equal one comes later)
                __syncthreads();
            }
        }
    };
    Eight<T> one[UNROLL], two[UNROLL];
    load(one, 0);
    for (int at = 0; at < count; at += 2 * turn) {  // (the next logits are on their way while these are taken)
        const int next = at + turn;
        if (next < count) load(two, next);
        take(one, at);
        if (next < count) {
            if (next + turn < count) load(one, next + turn);
            take(two, next);
        }
    }
    a = wave_join(a);
    if (lane == 0) wave_stats[wave] = a;
    __syncthreads();
    a = wave_join(lane < waves ? wave_stats[lane] : Stats{kLowest, 0.0f, 0.0f});
    if (p.parts == 1) {
        finish_row<T>(p, t, a, candidates.sorted);
    } else {
        const int64_t at = t * p.parts + blockIdx.x;
        if (threadIdx.x == 0) p.stats[at] = a;
        if constexpr (TOP)
            if ((int)threadIdx.x < p.top) p.best[at * p.top + threadIdx.x] = (int)threadIdx.x < candidates.count ? candidates.sorted[threadIdx.x] : 0;
    }
}

// Joins the parts of a row: 5 us, the latency of loads, two rounds of ranks and the selection.  Of the parts' alternatives only those matter that are not behind the last one of any part that has `top` of them, nor behind the
// top'th of the parts' first ones.
constexpr int kJoinThreads = 256, kMostParts = 64;
template <typename T> __global__ __launch_bounds__(kJoinThreads) void k_logprobs_join(LogprobArgs p)
{
    __shared__ Candidates<kMostParts * kMostTop> candidates;
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x % kWave;
    const uint64_t *all = p.best + t * p.parts * p.top;
    Stats a = lane < p.parts ? p.stats[t * p.parts + lane] : Stats{kLowest, 0.0f, 0.0f};
    if (p.top) {
        const int firsts = min((p.top + p.parts - 1) / p.parts, kWave / p.parts);
        const uint32_t one = lane < p.parts * firsts ? (uint32_t)(all[lane % p.parts * p.top + lane / p.parts] >> 32) : 0;
        uint32_t least = wave_max(lane < p.parts ? (uint32_t)(all[lane * p.top + p.top - 1] >> 32) : 0);
        least = max(least, of_rank(one, p.top - 1));
        if (threadIdx.x == 0) candidates.count = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < p.parts * p.top; i += kJoinThreads) {
            const uint64_t a = all[i];
            if (a >> 32 >= least && a) candidates.append(a);
        }
        __syncthreads();
        candidates.select(p.top);
    }
    a = wave_join(a);
    __syncthreads();
    finish_row<T>(p, t, a, candidates.sorted);
}

struct LogprobBackArgs {
    const void *logits;
    int64_t ldz, ldd, vocabulary;
    const void *ids;
    int32_t id_bytes;
    const float *lse, *entropy, *g_logp, *g_entropy;
    void *d_logits;
};

// The gradient.  p is exp(z - lse), and lse, in 32 bits, is off by half its last place, which p is then off by relative to itself: up to 2^-21, what the other roundings of z - lse
// come to, for |lse| below 16; for results of 16 bits, which are off by 2^-12 and more themselves, 2^-19 is let pass, for |lse| below 64.  Rows whose lse is larger have their largest logit and
// its sum taken again, as the forward call took them, and p from those: by one of the row's workgroups, which then takes all of the row (d_logits may be the logits, so that no other one may
// read what it writes).  us, such rows and others: 4096 x 32001 fp32 374 and 193, bf16 256 and 108; 64 x 50001 fp32 16 and 8; one row of 131072 27 and 8.
template <typename T> constexpr float kLseLimit = sizeof(T) == 4 ? 16.0f : 64.0f;

// below(z): z - lse
template <typename T, typename F>
__device__ __forceinline__ void logit_gradients(const Eight<T> &v, Eight<T> &out, int64_t col, int64_t id, float u, float w, float entropy, bool none, F below)
{
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float lp = below(v.get(i));
        const float prob = __builtin_amdgcn_exp2f(lp * kPerLog2);
        float g = prob * (u + (prob > 0.0f ? w * (lp + entropy) : 0.0f));
        g = col + i == id ? u - g : -g;
        if (none) g = u == u ? 0.0f : u;
        out.set(i, g);
    }
}

// Eight logits a thread.  Bound: HBM; 4096 x 32001 bf16 93 us, 5.6 TB/s read and written.
template <typename T, int THREADS> __global__ __launch_bounds__(THREADS) void k_logprobs_backward(LogprobBackArgs p)
{
    __shared__ Stats wave_stats[THREADS / kWave];
    const int64_t t = blockIdx.y;
    const T *z = static_cast<const T *>(p.logits) + t * p.ldz;
    T *d = static_cast<T *>(p.d_logits) + t * p.ldd;
    const int64_t id = p.ids ? id_at(p.ids, p.id_bytes, t) : -1;
    const float lse = p.lse[t], entropy = p.g_entropy ? p.entropy[t] : 0.0f, w = p.g_entropy ? p.g_entropy[t] : 0.0f;
    float u = id >= 0 && p.g_logp ? p.g_logp[t] : 0.0f;
    if (id >= p.vocabulary && p.g_logp) u = NAN;
    const bool none = lse == -INFINITY;
    const int64_t col = ((int64_t)blockIdx.x * THREADS + threadIdx.x) * 8, left = p.vocabulary - col;
    Eight<T> v, out;
    v.load_first(z + col, left);  // (on its way while lse is waited for; not used where another workgroup has the row)
    if (none || !(fabsf(lse) >= kLseLimit<T>)) {
        if (left <= 0) return;
        logit_gradients(v, out, col, id, u, w, entropy, none, [&](float z) { return z - lse; });
        out.store_first(d + col, left);
        return;
    }
    if (blockIdx.x != blockIdx.y % gridDim.x) return;  // (not the first one in every row: those may all be of one XCD)
    constexpr int kAhead = 2, kTurn = THREADS * 8;
    Stats a{kLowest, 0.0f, 0.0f};
    for (int64_t col = threadIdx.x * 8; col < p.vocabulary; col += kAhead * kTurn) {
        Eight<T> some[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; k++) some[k].load_first(z + col + k * kTurn, p.vocabulary - col - k * kTurn);
#pragma unroll
        for (int k = 0; k < kAhead; k++) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; i++) f[i] = col + k * kTurn + i < p.vocabulary ? some[k].get(i) : -INFINITY;
            add_eight(a, f);
        }
    }
    a = wave_join(a);
    if (threadIdx.x % kWave == 0) wave_stats[threadIdx.x / kWave] = a;
    __syncthreads();
    const int lane = threadIdx.x % kWave;
    a = wave_join(lane < THREADS / kWave ? wave_stats[lane] : Stats{kLowest, 0.0f, 0.0f});
    const float log_s = logf(a.s);
    for (int64_t col = threadIdx.x * 8; col < p.vocabulary; col += kAhead * kTurn) {
        Eight<T> some[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; k++) some[k].load_first(z + col + k * kTurn, p.vocabulary - col - k * kTurn);
#pragma unroll
        for (int k = 0; k < kAhead; k++) {
            logit_gradients(some[k], out, col + k * kTurn, id, u, w, entropy, false, [&](float z) { return z - a.m - log_s; });
            out.store_first(d + col + k * kTurn, p.vocabulary - col - k * kTurn);
        }
    }
}

// parts of a row: enough workgroups for the chip (one block each: 64 x 50001 in 8 parts of two blocks 22 us, in 13 of one 15), none of fewer than 4096 logits
int64_t parts_of(int64_t tokens, int64_t vocabulary)
{
    const int64_t most = (vocabulary + 4095) / 4096, wanted = (2048 + tokens - 1) / (tokens > 0 ? tokens : 1);
    const int64_t parts = wanted < most ? wanted : most;
    return parts < kMostParts ? parts : kMostParts;
}

int check_logits(int type, int64_t ldz, int64_t tokens, int64_t vocabulary)
{
    if (!is_type(type) || tokens < 0 || vocabulary < 1 || (tokens > 1 && ldz < vocabulary)) return HBP_ERR_INVALID_ARGUMENT;
    if (vocabulary > (int64_t(1) << 30) || tokens > (int64_t(1) << 31) - 512) return HBP_ERR_TOO_LARGE;
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
            const int64_t eights = (p.part + 7) / 8;
            const int threads = (int)(eights < kMostThreads ? (eights + kWave - 1) / kWave * kWave : kMostThreads);
            const bool longer = p.part > kMostThreads * 8;
            if (top) {
                if (longer) k_logprobs<T, true, 2><<<grid, threads, 0, st>>>(q);
                else k_logprobs<T, true, 1><<<grid, threads, 0, st>>>(q);
            } else {
                if (longer) k_logprobs<T, false, 2><<<grid, threads, 0, st>>>(q);
                else k_logprobs<T, false, 1><<<grid, threads, 0, st>>>(q);
            }
            HBP_HIP(hipGetLastError());
            if (p.parts > 1) {
                k_logprobs_join<T><<<dim3((unsigned)rows), kJoinThreads, 0, st>>>(q);
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
            auto go = [&](auto kernel, int threads) { kernel<<<dim3((unsigned)((vocabulary + threads * 8 - 1) / (threads * 8)), (unsigned)rows), threads, 0, (hipStream_t)stream>>>(p); };
            if (rows < 256) go(k_logprobs_backward<T, 1024>, 1024);  // (so that a row that is one workgroup's is not a quarter of a compute unit's)
            else go(k_logprobs_backward<T, 256>, 256);
            HBP_HIP(hipGetLastError());
        }
        return HBP_OK;
    });
}

}  // extern "C"
