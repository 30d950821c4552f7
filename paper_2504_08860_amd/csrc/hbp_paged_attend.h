// What the translation units of the attention over a paged cache share.
#pragma once

#include "hbp_paged.h"
#include "hbp_paged_split.h"

namespace hbp {

struct Attend {
    Paged c;
    const void *q;
    void *out;
    int64_t ldq, ldo;
    int32_t tokens, heads, group, most_new, window;
    float per;                 // scores to exponents of 2: |scale| / log 2, 1 where it is 0
    float cap_in, cap_out;     // with a cap: exponents are cap_out tanh(cap_in score); cap_out 0: none
    uint32_t keep, flip;       // of queries' bits, in both halves of a word: signs change where scale is negative, a scale of 0 leaves zeros
    Divider by_group;
    int32_t tile_rows;         // rows (a token's query heads of one head of keys lie together) that a workgroup takes at once
    int32_t places, aim, least, enough, whole;   // how tiles are split, see find_unit; of one head of keys
    int32_t slots;             // places for results of parts, of each head of keys
    float *partial;            // [slots][kv_heads][tile_rows][head_dim], sums of weights times values
    float2 *partial_stats;     // [slots][kv_heads][tile_rows]: the largest exponent, the sum of weights
    int64_t tiles, units;      // at most, of one head of keys
};

int launch_attend_f32(const Attend &a, hipStream_t st);
int launch_attend_f16(const Attend &a, hipStream_t st);
int launch_attend_bf16(const Attend &a, hipStream_t st);

// sum over the lanes up to each
__device__ __forceinline__ int32_t wave_running_sum(int32_t v)
{
    auto add = [&](auto control, auto rows) { v += __builtin_amdgcn_update_dpp(0, v, decltype(control)::value, decltype(rows)::value, 0xf, false); };
    using all = std::integral_constant<int, 0xf>;
    add(std::integral_constant<int, 0x111>(), all());   // row_shr 1, 2, 4, 8: within rows of 16
    add(std::integral_constant<int, 0x112>(), all());
    add(std::integral_constant<int, 0x114>(), all());
    add(std::integral_constant<int, 0x118>(), all());
    add(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());   // the last of a row to the next one, for rows 1 and 3
    add(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());   // that of row 1 to rows 2 and 3
    return v;
}

// A part of a tile: the rows and the positions that a workgroup takes.
struct Unit {
    int32_t sequence, tile, part, parts, slot;   // slot: of the tile's first part
    int32_t first_token, rows;                   // of the sequence: its first row in q, how many (row, head) rows it has in all
    int64_t first_position;                      // of its first new token
    int32_t low, high, size;                     // positions that the tile's rows see, from a multiple of kStep on; a part's share
};

// Finds a unit (or, BY_TILE, a tile) by its number among those of one head of keys: by the whole workgroup, some neighbouring sequences a thread.  How tiles are split is
// decided here, from the lengths that the device holds: into parts of about the same length.  There are to be as many as the chip has places for at once (`places`), so that all of them are busy, but
// for that none is cut shorter than `least`; beyond `enough` positions they are cut finer, into up to `aim`, which evens out what the places get.  Tiles of up to
// `whole` positions are not split: joining their parts takes as long.
// Up to 64 sequences each wavefront finds its own, a lane a sequence; more are dealt to the workgroup's threads.  (256 sequences, 64 of them at a time, by each wavefront: 8 us, of loads that wait for
// each other.)
template <bool BY_TILE, int THREADS> __device__ __forceinline__ bool find_unit(const Attend &a, int32_t number, Unit &x)
{
    constexpr int kWaves = THREADS / kWave;
    __shared__ int32_t work_of[kWaves][3], units_of[kWaves], slots_of[kWaves], found[9];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    struct Sequence {
        int32_t first, count, taken, length, tiles, span;
    };
    const int32_t tile_tokens = (a.tile_rows - 2 + a.group) / a.group + 1;   // that a tile's rows are of, at most
    auto get = [&](int32_t s) {
        Sequence q{0, 0, 0, 0, 0, 0};
        if (s < a.c.sequences) {
            const int32_t begin = a.c.starts[s], end = a.c.starts[s + 1];
            q.length = a.c.lengths[s];
            q.first = begin;
            if (begin >= 0 && end > begin && end <= a.tokens) {
                q.count = end - begin;
                q.taken = min(q.count, a.most_new);
                q.tiles = (int32_t)(((int64_t)q.taken * a.group + a.tile_rows - 1) / a.tile_rows);
                q.span = max(0, min(q.length, a.c.capacity));
                if (a.window) q.span = (int32_t)min((int64_t)q.span, (int64_t)a.window + tile_tokens);
            }
        }
        return q;
    };
    const bool few = a.c.sequences <= kWave;
    const int32_t each = few ? 1 : (a.c.sequences + THREADS - 1) / THREADS, mine = few ? lane : (int32_t)threadIdx.x * each;
    const Sequence own = get(mine);
    int64_t work = (int64_t)own.tiles * own.span;
    for (int32_t i = 1; i < each; i++) {
        const Sequence q = get(mine + i);
        work += (int64_t)q.tiles * q.span;
    }
    // the sum in three pieces of 24 bits, so that it is the same in every kernel in whatever order it is added
    int32_t piece[3] = {(int32_t)(work & 0xffffff), (int32_t)(work >> 24 & 0xffffff), (int32_t)(work >> 48)};   // (64 lanes' sums are below 2^30; those of wavefronts are added in 64 bits)
#pragma unroll
    for (int i = 0; i < 3; i++) piece[i] = wave_reduce(piece[i], [](int32_t p, int32_t q) { return p + q; });
    auto whole_of = [](const int32_t (&p)[3]) { return p[0] + ((int64_t)p[1] << 24) + ((int64_t)p[2] << 48); };
    int64_t all_work = 0;
    if (few) {
        all_work = whole_of(piece);
    } else {
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < 3; i++) work_of[wave][i] = piece[i];
        if (threadIdx.x == 0) found[0] = -1;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; w++) all_work += whole_of(work_of[w]);
    }
    int32_t length = part_length((double)all_work, a.places, a.aim, a.enough, a.least);
    // (what the last part of each tile is shorter by makes them more than the places: a second turn of the chip for a few)
    if (few && length < a.enough)
        for (int i = 0; i < 4; i++) {
            const int32_t all = wave_reduce(own.tiles * part_count(own.span, length, a.whole), [](int32_t p, int32_t q) { return p + q; });
            const int64_t longer = ((int64_t)length * all / a.places + kStep) / kStep * kStep;
            if (all <= a.places || longer > a.enough) break;
            length = (int32_t)longer;
        }
    auto parts_of = [&](const Sequence &q) { return part_count(q.span, length, a.whole); };
    auto add = [&](const Sequence &q, int32_t &units, int32_t &slots) {
        const int32_t parts = parts_of(q);
        units += BY_TILE ? q.tiles : q.tiles * parts;
        slots += parts > 1 ? q.tiles * parts : 0;
    };
    int32_t units = 0, slots = 0;
    add(own, units, slots);
    for (int32_t i = 1; i < each; i++) add(get(mine + i), units, slots);
    const int32_t upto = wave_running_sum(units), slots_upto = wave_running_sum(slots);
    int32_t before = upto - units, slots_before = slots_upto - slots;
    if (!few) {
        if (lane == kWave - 1) {
            units_of[wave] = upto;
            slots_of[wave] = slots_upto;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; w++)
            if (w < wave) {
                before += units_of[w];
                slots_before += slots_of[w];
            }
    }
    const bool is_mine = number >= before && number < before + units;
    Sequence q = own;
    int32_t at = mine;
    if (!few && is_mine) {
        int32_t next = 0, next_slots = 0;
        add(q, next, next_slots);
        while (number >= before + next) {
            before += next;
            slots_before += next_slots;
            q = get(++at);
            next = next_slots = 0;
            add(q, next, next_slots);
        }
    }
    const int32_t parts = parts_of(q), local = number - before;
    const int32_t tile = q.tiles - 1 - (BY_TILE ? local : local / parts);   // (the latest tiles of a prompt see the most and are taken first)
    int32_t values[9] = {at, tile, BY_TILE ? 0 : local % parts, parts, slots_before + tile * parts, q.first, q.taken, q.length, q.count};
    if (few) {
        const uint64_t lanes = __ballot(is_mine);
        if (!lanes) return false;
        const int owner = __builtin_ctzll(lanes);
#pragma unroll
        for (int i = 0; i < 9; i++) values[i] = __builtin_amdgcn_readlane(values[i], owner);
    } else {
        if (is_mine)
#pragma unroll
            for (int i = 0; i < 9; i++) found[i] = values[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 9; i++) values[i] = __builtin_amdgcn_readfirstlane(found[i]);
        if (values[0] < 0) return false;
    }
    x.sequence = values[0];
    x.tile = values[1];
    x.part = values[2];
    x.parts = values[3];
    x.slot = values[4];
    x.first_token = values[5];
    if (x.parts > 1 && (x.slot < 0 || x.slot > a.slots - x.parts)) return false;   // (more than the host counted: only where `starts` does not ascend)
    x.rows = values[6] * a.group;
    x.first_position = (int64_t)values[7] - values[8];
    const int32_t row = x.tile * a.tile_rows, last = min(row + a.tile_rows, x.rows) - 1;
    const int64_t p0 = x.first_position + a.by_group.divide(row), p1 = x.first_position + a.by_group.divide(last);
    x.low = (int32_t)max((int64_t)0, a.window ? p0 - a.window + 1 : 0) / kStep * kStep;
    x.high = (int32_t)max((int64_t)0, min(p1 + 1, (int64_t)a.c.capacity));
    const int32_t span = max(0, x.high - x.low);
    x.size = ((span + x.parts - 1) / x.parts + kStep - 1) / kStep * kStep;
    return true;
}

}  // namespace hbp
