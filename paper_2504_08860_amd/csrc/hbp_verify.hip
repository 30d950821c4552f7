// Drafted tokens against the target's probabilities, and the token drawn behind those that stand (hbp_verify_drafts).
//
// What comes out are whole numbers: an index is off where a running sum lies on the wrong side of a border, and over a hundred thousand tokens of which each
// has its border, sums in 32 bits would be so in one of some hundred draws.  So exponentials and sums are held in 64 bits from the logits on.
#include "hbp_paged.h"

#include <algorithm>

namespace hbp {
namespace {

// A part of a row: its largest logit (-inf: nothing is left, or NaN), the lowest index of that, and the sum of exp((z - largest) / temperature).
struct RowPart {
    double sum;
    float largest;
    int32_t first;
};

constexpr int kThreads = 256, kWaves = kThreads / kWave, kDrawThreads = 256;
constexpr int kTurn = 16 * kWave, kPart = 2 * kTurn, kMostParts = kWave;   // logits that a wavefront takes at once, and of a part; rows of more than kMostParts such have longer parts

struct VerifyArgs {
    const void *logits;
    const void *ids;
    const float *uniforms, *temperature, *draft_probs;
    const int32_t *starts;
    int32_t *new_ids, *accepted;
    RowPart *stats;      // [rows][parts]
    RowPart *decided;    // [sequences], where there are draft_probs: the row that the new token is drawn from, its parts joined
    int32_t *decided_row;
    double *weights;     // [sequences][parts], the same
    int64_t ldz, ldp;
    int32_t rows, vocabulary, sequences, id_bytes, parts, part;
};

// 2^(y / 64) for y <= 0, to some 2^-44 of it: y is a whole number of sixty-fourths, of which the last six bits choose one of sixty-four powers (in LDS) and the others are the
// exponent, and a rest x log 2 of at most log 2 / 128, of whose series the first missing term is 4e-14.  The whole number comes out of the last bits of a sum with 3 * 2^51.
constexpr double kFar = -64000.0;   // 2^-1000, and 0 for what is further down
struct Table {
    double of[64];
    constexpr Table() : of{}
    {
        for (int i = 0; i < 64; i++) {
            const double x = i * (0.69314718055994531 / 64);
            double term = 1.0, sum = 0.0;
            for (int k = 1; k < 30; k++) {
                sum += term;
                term *= x / k;
            }
            of[i] = sum;
        }
    }
};
__device__ const Table kTable;
struct Powers {
    double of[64];
    __device__ __forceinline__ void set()   // (a barrier follows)
    {
        if (threadIdx.x < 64) of[threadIdx.x] = kTable.of[threadIdx.x];
    }
    __device__ __forceinline__ double power_near(double y) const   // y > kFar, or NaN, which stays
    {
        constexpr double c1 = 0.69314718055994531 / 64, c2 = c1 * c1 / 2, c3 = c2 * c1 / 3, c4 = c3 * c1 / 4, kWhole = 6755399441055744.0;
        const double sum = y + kWhole, r = y - (sum - kWhole);
        const int32_t whole = (int32_t)__builtin_bit_cast(uint64_t, sum);
        const double v = fma(fma(fma(fma(c4, r, c3), r, c2), r, c1), r, 1.0) * of[whole & 63];
        const uint64_t bits = __builtin_bit_cast(uint64_t, v);
        const uint32_t high = (uint32_t)(bits >> 32) + ((uint32_t)(whole & ~63) << 14);   // (the exponent's bits begin at 20 of these; a NaN's sum ends in zeros)
        return __builtin_bit_cast(double, (uint64_t)high << 32 | (uint32_t)bits);
    }
    __device__ __forceinline__ double power(double y) const   // NaN gives 0
    {
        const double e = power_near(y);
        return y > kFar ? e : 0.0;
    }
};

// what a difference of logits is multiplied by to be sixty-fourths of an exponent of 2: NaN where the temperature is none
__device__ __forceinline__ double per_logit(float temperature)
{
    constexpr double kPerLog2 = 64 * 1.4426950408889634;
    if (temperature == 0.0f) return kPerLog2;
    return temperature > 0.0f ? kPerLog2 / (double)temperature : (double)NAN;
}
// exp((z - largest) / temperature); per is a number, and NaN is looked for elsewhere
__device__ __forceinline__ double exponential(const Powers &powers, float z, float largest, double per)
{
    return powers.power(((double)z - (double)largest) * per);   // (0 for a masked one, also where per is 0)
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ double wave_running_sum(double v)   // of the lanes up to each
{
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const double below = __shfl_up(v, d);
        v += lane >= d ? below : 0.0;
    }
    return v;
}

// Eight logits from column `col` on; behind the end -inf.
template <typename T> __device__ __forceinline__ void load_logits(const T *z, int32_t col, int32_t end, float (&f)[8])
{
    Eight<T> v;
    v.load_first(z + col, end - col);
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = col + i < end ? v.get(i) : -INFINITY;
}

// Sums over parts of rows, a wavefront a part: its logits stay in registers between the largest one and the sum, the next ones on their way.  Bound: the vector unit, 11 instructions in 64 bits
// and 8 others a logit where all of a turn's logits are near enough to the largest to count and none is behind the end; and what a wavefront does beside that, which was as much with 16 logits a lane.
// 512 rows of 50001 fp32 logits 21.3 us, 4.8 TB/s; 1024 of 32001 fp16 24.8 us; 5 of 131072 3.4 us.
template <typename T> __global__ __launch_bounds__(kThreads) void k_verify_rows(VerifyArgs a, int32_t first_row)
{
    constexpr int kEights = kTurn / kWave / 8;
    __shared__ Powers powers;
    const int lane = threadIdx.x % kWave;
    const int32_t row = first_row + blockIdx.y, part = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + threadIdx.x / kWave);
    const int32_t begin = min(part * a.part, a.vocabulary), end = min(begin + a.part, a.vocabulary);
    const T *z = static_cast<const T *>(a.logits) + (int64_t)row * a.ldz;
    Eight<T> next[kEights];
    auto load = [&](int32_t from) {
#pragma unroll
        for (int k = 0; k < kEights; k++) {
            const int32_t col = from + (k * kWave + lane) * 8;
            if (from + kTurn <= end) next[k].load(z + col);
            else next[k].load_first(z + col, end - col);
        }
    };
    load(begin);
    powers.set();
    float temperature = 1.0f;
    if (a.temperature) {
        const int32_t s = __builtin_amdgcn_readfirstlane(sequence_of(a.starts, a.sequences, row));
        if (s < a.sequences) temperature = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(a.temperature[s])));
    }
    const double per = per_logit(temperature);
    __syncthreads();   // (the powers)
    float largest = -INFINITY;
    int32_t first = a.vocabulary;
    double sum = 0.0;
    bool odd = false;   // NaN
    for (int32_t from = begin; from < end; from += kTurn) {
        float f[kEights][8], m = largest, low = INFINITY;
#pragma unroll
        for (int k = 0; k < kEights; k++)
#pragma unroll
            for (int i = 0; i < 8; i++) f[k][i] = next[k].get(i);
        if (from + kTurn > end)
#pragma unroll
            for (int k = 0; k < kEights; k++)
#pragma unroll
                for (int i = 0; i < 8; i++) f[k][i] = from + (k * kWave + lane) * 8 + i < end ? f[k][i] : -INFINITY;
        if (from + kTurn < end) load(from + kTurn);
#pragma unroll
        for (int k = 0; k < kEights; k++)
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                asm("v_max3_f32 %0, %1, %2, %0" : "+v"(m) : "v"(f[k][i]), "v"(f[k][i + 1]));   // (fmaxf would make each value canonical first; NaN is passed over)
                asm("v_min3_f32 %0, %1, %2, %0" : "+v"(low) : "v"(f[k][i]), "v"(f[k][i + 1]));
            }
        const float top = hbp::wave_max(m);
        if (temperature == 0.0f) {
            int32_t at = a.vocabulary;
#pragma unroll
            for (int k = kEights - 1; k >= 0; k--)
#pragma unroll
                for (int i = 7; i >= 0; i--) {
                    odd |= f[k][i] != f[k][i];
                    at = f[k][i] == top ? from + (k * kWave + lane) * 8 + i : at;
                }
            at = (int32_t)~hbp::wave_max(~(uint32_t)at);   // (the lowest one)
            if (top > largest) first = at;
        } else {
            if (top > largest) sum *= exponential(powers, largest, top, per);
            const bool near = ((double)low - (double)top) * per > kFar;
            if (__ballot(!near) == 0) {
#pragma unroll
                for (int k = 0; k < kEights; k++)
#pragma unroll
                    for (int i = 0; i < 8; i++) sum += powers.power_near(((double)f[k][i] - (double)top) * per);
            } else {
#pragma unroll
                for (int k = 0; k < kEights; k++)
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        odd |= f[k][i] != f[k][i];
                        sum += exponential(powers, f[k][i], top, per);
                    }
            }
        }
        largest = top;
    }
    sum = wave_sum(odd ? (double)NAN : sum);
    if (lane == 0 && part < a.parts) {
        if (temperature == 0.0f && sum == 0.0) sum = largest > -INFINITY ? 1.0 : 0.0;
        if (largest == INFINITY || !(temperature >= 0.0f)) sum = NAN;
        a.stats[(int64_t)row * a.parts + part] = RowPart{sum, largest, first};
    }
}

// A whole row, from its parts, by a wavefront
__device__ __forceinline__ RowPart join_parts(const VerifyArgs &a, const Powers &powers, int32_t row, double per)
{
    const int lane = threadIdx.x % kWave;
    RowPart mine{0.0, -INFINITY, a.vocabulary};
    if (lane < a.parts) mine = a.stats[(int64_t)row * a.parts + lane];
    RowPart all;
    all.largest = hbp::wave_max(mine.largest);
    all.first = (int32_t)~hbp::wave_max(mine.largest == all.largest ? ~(uint32_t)mine.first : 0u);
    // (a part whose sum is NaN keeps it, whatever its largest logit is)
    all.sum = wave_sum(mine.sum == 0.0 ? 0.0 : mine.sum * exponential(powers, mine.largest, all.largest, per) + (mine.sum != mine.sum ? mine.sum : 0.0));
    return all;
}

__device__ __forceinline__ int64_t id_of(const VerifyArgs &a, int32_t row)
{
    return a.id_bytes == 8 ? static_cast<const int64_t *>(a.ids)[row] : static_cast<const int32_t *>(a.ids)[row];
}

// The first row of begin..end-1 whose draft does not stand (end - 1 where all do), by a workgroup, a wavefront a row; and that row's parts joined, in every thread
template <typename T, int THREADS>
__device__ __forceinline__ int32_t first_to_fall(const VerifyArgs &a, const Powers &powers, int32_t begin, int32_t end, float temperature, double per, RowPart &all)
{
    constexpr int kWaves = THREADS / kWave;
    __shared__ int32_t falls[kWaves];
    __shared__ RowPart joined[kWaves];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    for (int32_t from = begin;; from += kWaves) {
        const int32_t row = from + wave;
        bool stands = true;
        RowPart r{0.0, -INFINITY, 0};
        if (row < end) {
            const int64_t d = row + 1 < end ? id_of(a, row + 1) : -1;
            r = join_parts(a, powers, row, per);
            stands = false;   // (the last row's draft, which is none, never does)
            if (d >= 0 && d < a.vocabulary && r.sum > 0.0) {
                const double q = a.draft_probs ? (double)a.draft_probs[(int64_t)row * a.ldp + d] : 1.0;
                const double p = temperature == 0.0f ? (d == r.first ? 1.0 : 0.0)
                                                     : exponential(powers, to_f32(static_cast<const T *>(a.logits)[(int64_t)row * a.ldz + d]), r.largest, per) / r.sum;
                stands = (double)a.uniforms[row] * q < p;
            }
        }
        __syncthreads();
        if (lane == 0) {
            falls[wave] = stands ? end : row;
            joined[wave] = r;
        }
        __syncthreads();
        int32_t least = end;
#pragma unroll
        for (int w = 0; w < kWaves; w++) least = min(least, falls[w]);
        if (least < end) {
            all = joined[least - from];
            return least;
        }
    }
}

// What tokens `col`.. of eight are drawn by: max(p - q, 0), or p (as exponentials, or 1 at the largest) without the draft `d` where there are no draft_probs.
template <typename T, bool DIFFERENCE>
__device__ __forceinline__ void weights_of(const VerifyArgs &a, const Powers &powers, int32_t row, int32_t col, int32_t end, const RowPart &all, double inverse, float temperature, double per,
                                           int64_t d, double (&w)[8])
{
    float f[8];
    load_logits(static_cast<const T *>(a.logits) + (int64_t)row * a.ldz, col, end, f);
    Eight<float> q;
    if constexpr (DIFFERENCE) q.load_first(a.draft_probs + (int64_t)row * a.ldp + col, end - col);
    const int32_t gone = d >= col && d < col + 8 ? (int32_t)(d - col) : -1;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        double e = temperature == 0.0f ? (col + i == all.first ? 1.0 : 0.0) : exponential(powers, f[i], all.largest, per);
        if constexpr (DIFFERENCE) {
            const double p = temperature == 0.0f ? e : e * inverse;
            e = col + i < end ? fmax(p - (double)q.get(i), 0.0) : 0.0;
            if (q.get(i) != q.get(i)) e = NAN;
        } else if (col + i >= end || i == gone) {
            e = 0.0;
        }
        w[i] = e;
    }
}

// sums over parts of max(p - q, 0), of the row whose draft does not stand, a wavefront a part.  Bound: the chain that finds the row (ids, parts, exponentials), which every workgroup
// walks by itself for a launch less: 5.7 us for one sequence, 13.6 for 256 of 4 rows of 32001.
template <typename T> __global__ __launch_bounds__(kThreads) void k_verify_differences(VerifyArgs a, int32_t first_sequence)
{
    __shared__ Powers powers;
    const int32_t s = first_sequence + blockIdx.y, begin = a.starts[s], end = a.starts[s + 1];
    if (begin < 0 || end <= begin || end > a.rows) return;
    powers.set();
    const float temperature = a.temperature ? a.temperature[s] : 1.0f;
    const double per = per_logit(temperature);
    __syncthreads();
    RowPart all;
    const int32_t row = first_to_fall<T, kThreads>(a, powers, begin, end, temperature, per, all);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.decided[s] = all;
        a.decided_row[s] = row;
    }
    const int32_t part = blockIdx.x * kWaves + threadIdx.x / kWave;
    if (row == end - 1 || part >= a.parts) return;
    const double inverse = 1.0 / all.sum;
    const int32_t from = part * a.part, to = min(from + a.part, a.vocabulary);
    double sum = 0.0;
#pragma unroll 2
    for (int32_t col = from + threadIdx.x % kWave * 8; col < to; col += kWave * 8) {
        double w[8];
        weights_of<T, true>(a, powers, row, col, to, all, inverse, temperature, per, -1, w);
#pragma unroll
        for (int i = 0; i < 8; i++) sum += w[i];
    }
    sum = wave_sum(sum);
    if (threadIdx.x % kWave == 0) a.weights[(int64_t)s * a.parts + part] = sum;
}

// The drafts that stand and the new token, a workgroup a sequence: the part that the drawn place is in, by the parts' sums, then the token in it.  A chain of loads: 3.4 us for one
// sequence, 5.6 for 256, 7.4 for 64 that look for the row too.  256 threads take a part of 2048 tokens at once.
template <typename T> __global__ __launch_bounds__(kDrawThreads) void k_verify_draw(VerifyArgs a, int32_t first_sequence)
{
    constexpr int kDrawWaves = kDrawThreads / kWave;
    __shared__ double wave_sums[kDrawWaves];
    __shared__ int32_t found_by[kDrawWaves], latest_by[kDrawWaves];
    __shared__ Powers powers;
    const int32_t s = first_sequence + blockIdx.x, begin = a.starts[s], end = a.starts[s + 1];
    if (begin < 0 || end <= begin || end > a.rows) {
        if (threadIdx.x == 0) a.accepted[s] = 0;
        return;
    }
    powers.set();
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const float temperature = a.temperature ? a.temperature[s] : 1.0f;
    const double per = per_logit(temperature);
    __syncthreads();
    RowPart all;
    int32_t row;
    if (a.draft_probs) {
        all = a.decided[s];
        row = a.decided_row[s];
    } else {
        row = first_to_fall<T, kDrawThreads>(a, powers, begin, end, temperature, per, all);
    }
    const bool fell = row < end - 1;
    int64_t d = fell && !a.draft_probs ? id_of(a, row + 1) : -1;
    bool difference = fell && a.draft_probs;
    // the parts' sums of weights, a lane a part
    double part = 0.0, total = 0.0;
    if (difference) {
        if (lane < a.parts) part = a.weights[(int64_t)s * a.parts + lane];
        total = wave_sum(part);
        if (!(total > 0.0)) difference = false;   // (nothing is left of p - q: p)
    }
    auto of_p = [&](int64_t without) {
        const RowPart mine = lane < a.parts ? a.stats[(int64_t)row * a.parts + lane] : RowPart{0.0, -INFINITY, a.vocabulary};
        const bool has = without >= 0 && without < a.vocabulary && without / a.part == lane;
        if (temperature == 0.0f) {
            part = lane == all.first / a.part && all.first != without ? 1.0 : 0.0;
        } else {
            part = mine.sum > 0.0 ? mine.sum * exponential(powers, mine.largest, all.largest, per) : 0.0;
            if (has) part = fmax(part - exponential(powers, to_f32(static_cast<const T *>(a.logits)[(int64_t)row * a.ldz + without]), all.largest, per), 0.0);
        }
        total = wave_sum(part);
    };
    if (!difference) {
        of_p(d);
        if (!(total > 0.0) && d >= 0) {   // (the draft was all there is)
            d = -1;
            of_p(-1);
        }
    }
    int32_t token = -1;
    if (all.sum > 0.0 && total > 0.0) {   // (the same in every thread)
        const double wanted = (double)a.uniforms[end - 1] * total;
        const double running = wave_running_sum(part);
        uint64_t over = __ballot(running > wanted && part > 0.0);
        const uint64_t some = __ballot(part > 0.0);
        if (!over) over = 1ull << (63 - __builtin_clzll(some));   // (roundings: the last one with a weight)
        const int which = __builtin_ctzll(over);
        const double before = __shfl(running, which) - __shfl(part, which);
        const double left = wanted - before, inverse = 1.0 / all.sum;
        const int32_t from = which * a.part, to = min(from + a.part, a.vocabulary);
        double base = 0.0;
        int32_t last = -1;   // the last token with a weight so far
        for (int32_t at = from; at < to && token < 0; at += kDrawThreads * 8) {
            const int32_t col = at + threadIdx.x * 8;
            double w[8];
            if (col < to) {
                if (difference) weights_of<T, true>(a, powers, row, col, to, all, inverse, temperature, per, -1, w);
                else weights_of<T, false>(a, powers, row, col, to, all, inverse, temperature, per, d, w);
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) w[i] = 0.0;
            }
            double mine = 0.0;
#pragma unroll
            for (int i = 0; i < 8; i++) mine += w[i];
            const double upto = wave_running_sum(mine);
            __syncthreads();
            if (lane == kWave - 1) wave_sums[wave] = upto;
            __syncthreads();
            double below = base + upto - mine;
#pragma unroll
            for (int k = 0; k < kDrawWaves; k++) {
                if (k < wave) below += wave_sums[k];
                base += wave_sums[k];
            }
            int32_t found = 0x7fffffff, latest = -1;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                below += w[i];
                if (w[i] > 0.0) {
                    latest = col + i;
                    if (below > left) found = min(found, col + i);
                }
            }
            const int32_t wave_found = (int32_t)~hbp::wave_max(~(uint32_t)found), wave_latest = (int32_t)hbp::wave_max((uint32_t)(latest + 1)) - 1;
            if (lane == 0) {
                found_by[wave] = wave_found;
                latest_by[wave] = wave_latest;
            }
            __syncthreads();
            found = 0x7fffffff;
#pragma unroll
            for (int k = 0; k < kDrawWaves; k++) {
                found = min(found, found_by[k]);
                last = max(last, latest_by[k]);
            }
            if (found != 0x7fffffff) token = found;
        }
        if (token < 0) token = last;
    }
    for (int32_t r = begin + threadIdx.x; r < end; r += kDrawThreads) a.new_ids[r] = r < row ? (int32_t)id_of(a, r + 1) : r == row ? token : -1;
    if (threadIdx.x == 0) a.accepted[s] = row - begin;
}

__global__ void k_verify_nothing(int32_t *accepted, int32_t sequences)
{
    for (int32_t s = blockIdx.x * blockDim.x + threadIdx.x; s < sequences; s += gridDim.x * blockDim.x) accepted[s] = 0;
}

// logits of a part: whole turns, so that only the last part of a row ends inside one
int32_t part_of(int64_t vocabulary)
{
    const int64_t part = ((vocabulary + kMostParts - 1) / kMostParts + kTurn - 1) / kTurn * kTurn;
    return (int32_t)std::max<int64_t>(part, kPart);
}
int32_t parts_of(int64_t vocabulary) { return (int32_t)((vocabulary + part_of(vocabulary) - 1) / part_of(vocabulary)); }

}  // namespace
}  // namespace hbp

extern "C" {

int hbp_verify_drafts_workspace(int64_t rows, int64_t vocabulary, int64_t sequences, size_t *bytes)
{
    using namespace hbp;
    if (rows < 0 || vocabulary < 1 || sequences < 0 || !bytes) return HBP_ERR_INVALID_ARGUMENT;
    if (rows > (int64_t(1) << 30) || vocabulary > (int64_t(1) << 30) || sequences > (int64_t(1) << 24)) return HBP_ERR_TOO_LARGE;
    *bytes = rows && sequences ? (size_t)parts_of(vocabulary) * ((size_t)rows * sizeof(RowPart) + (size_t)sequences * sizeof(double)) + (size_t)sequences * (sizeof(RowPart) + sizeof(int32_t)) : 0;
    return HBP_OK;
}

int hbp_verify_drafts(int type, const void *logits, int64_t ldz, int64_t rows, int64_t vocabulary, const void *ids, int id_bytes, const float *uniforms,
                      const int32_t *starts, int64_t sequences, const float *temperature, const float *draft_probs, int64_t ldp, int32_t *new_ids,
                      int32_t *accepted, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace hbp;
    size_t need = 0;
    int rc = hbp_verify_drafts_workspace(rows, vocabulary, sequences, &need);
    if (rc != HBP_OK) return rc;
    if (!is_type(type)) return HBP_ERR_INVALID_ARGUMENT;
    if (sequences == 0) return HBP_OK;
    if (!accepted || !aligned(accepted, 4)) return HBP_ERR_INVALID_ARGUMENT;
    hipStream_t st = (hipStream_t)stream;
    if (rows > 0) {
        if (!logits || !ids || !uniforms || !starts || !new_ids || (id_bytes != 4 && id_bytes != 8)) return HBP_ERR_INVALID_ARGUMENT;
        if (!aligned(logits, type_bytes(type)) || !aligned(ids, id_bytes)) return HBP_ERR_INVALID_ARGUMENT;
        for (const void *p : {(const void *)uniforms, (const void *)starts, (const void *)temperature, (const void *)draft_probs, (const void *)new_ids})
            if (!aligned(p, 4)) return HBP_ERR_INVALID_ARGUMENT;
        if (rows > 1 && (ldz < vocabulary || (draft_probs && ldp < vocabulary))) return HBP_ERR_INVALID_ARGUMENT;
        if (!workspace || workspace_bytes < need || !aligned(workspace, 256)) return HBP_ERR_INVALID_ARGUMENT;
    }
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    if (rows == 0) {
        k_verify_nothing<<<dim3((unsigned)std::min<int64_t>((sequences + 255) / 256, 1024)), 256, 0, st>>>(accepted, (int32_t)sequences);
        HBP_HIP(hipGetLastError());
        return HBP_OK;
    }
    VerifyArgs a{};
    a.logits = logits; a.ldz = ldz; a.rows = (int32_t)rows; a.vocabulary = (int32_t)vocabulary;
    a.ids = ids; a.id_bytes = id_bytes; a.uniforms = uniforms; a.starts = starts; a.sequences = (int32_t)sequences;
    a.temperature = temperature; a.draft_probs = draft_probs; a.ldp = ldp;
    a.new_ids = new_ids; a.accepted = accepted;
    a.parts = parts_of(vocabulary);
    a.part = part_of(vocabulary);
    a.stats = static_cast<RowPart *>(workspace);
    a.decided = a.stats + rows * a.parts;
    a.weights = reinterpret_cast<double *>(a.decided + sequences);
    a.decided_row = reinterpret_cast<int32_t *>(a.weights + sequences * a.parts);
    return by_type(type, [&](auto t) -> int {
        using T = decltype(t);
        const unsigned across = (unsigned)((a.parts + kWaves - 1) / kWaves);
        constexpr int64_t kMost = 32768;   // of one launch: the grid's second dimension ends at 65535
        for (int64_t at = 0; at < rows; at += kMost) {
            k_verify_rows<T><<<dim3(across, (unsigned)std::min(rows - at, kMost)), kThreads, 0, st>>>(a, (int32_t)at);
            HBP_HIP(hipGetLastError());
        }
        for (int64_t at = 0; at < sequences; at += kMost) {
            const unsigned count = (unsigned)std::min(sequences - at, kMost);
            if (draft_probs) {
                k_verify_differences<T><<<dim3(across, count), kThreads, 0, st>>>(a, (int32_t)at);
                HBP_HIP(hipGetLastError());
            }
            k_verify_draw<T><<<dim3(count), kDrawThreads, 0, st>>>(a, (int32_t)at);
            HBP_HIP(hipGetLastError());
        }
        return HBP_OK;
    });
}

}  // extern "C"
