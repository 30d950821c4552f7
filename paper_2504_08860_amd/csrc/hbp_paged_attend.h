// What the translation units of the attention over a paged cache share.
#pragma once

#include "hbp_paged.h"

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
    Divider by_group, by_kv_heads;
    int32_t tile_rows;         // rows (a token's query heads of one head of keys lie together) that a workgroup takes at once
    int32_t aim, least;        // parts of all tiles of one head of keys, about, and positions that a part has at least
    int32_t slots;             // places for results of parts, of each head of keys
    float *partial;            // [slots][kv_heads][tile_rows][head_dim], sums of weights times values
    float2 *partial_stats;     // [slots][kv_heads][tile_rows]: the largest exponent, the sum of weights
    int64_t tiles;             // at most, of one head of keys
};

constexpr int kStep = 32;   // positions that a matrix instruction takes at once; parts begin at multiples of it

int launch_attend_f32(const Attend &a, hipStream_t st);
int launch_attend_f16(const Attend &a, hipStream_t st);
int launch_attend_bf16(const Attend &a, hipStream_t st);

// A part of a tile: the rows and the positions that a workgroup takes.
struct Unit {
    int32_t sequence, tile, part, parts, slot;   // slot: of the tile's first part
    int32_t first_token, rows;                   // of the sequence: its first row in q, how many (row, head) rows it has in all
    int64_t first_position;                      // of its first new token
    int32_t low, high, size;                     // positions that the tile's rows see, from a multiple of kStep on; a part's share
};

// Finds a unit (or, BY_TILE, a tile) by its number among those of one head of keys: every wavefront for itself, a lane a sequence.  How tiles are split is
// decided here, from the lengths that the device holds: into parts of about the same length, as many in all as `aim` says, and none of fewer than `least` positions.
template <bool BY_TILE> __device__ __forceinline__ bool find_unit(const Attend &a, int32_t number, Unit &x)
{
    const int lane = threadIdx.x % kWave;
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
    Sequence mine = get(lane);
    float total = wave_reduce((float)mine.tiles * (float)mine.span, [](float p, float q) { return p + q; });
    for (int32_t from = kWave; from < a.c.sequences; from += kWave) {
        const Sequence q = get(from + lane);
        total += wave_reduce((float)q.tiles * (float)q.span, [](float p, float q) { return p + q; });
    }
    const float share = fminf(ceilf(total / (float)a.aim), 1073741824.0f);
    const int32_t length = (max(a.least, __builtin_amdgcn_readfirstlane((int32_t)share)) + kStep - 1) / kStep * kStep;
    int32_t units = 0, slots = 0;   // of the sequences before
    for (int32_t from = 0; from < a.c.sequences; from += kWave) {
        if (from) mine = get(from + lane);
        const int32_t parts = max(1, (int32_t)((mine.span + length - 1) / length));
        const int32_t my_units = BY_TILE ? mine.tiles : mine.tiles * parts, my_slots = parts > 1 ? mine.tiles * parts : 0;
        int32_t upto = my_units, slots_upto = my_slots;
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const int32_t u = __shfl_up(upto, d), v = __shfl_up(slots_upto, d);
            upto += lane >= d ? u : 0;
            slots_upto += lane >= d ? v : 0;
        }
        const int32_t all = __builtin_amdgcn_readlane(upto, kWave - 1);
        if (number < units + all) {
            const int at = __builtin_ctzll(__ballot(number < units + upto));
            auto of = [&](int32_t v) { return __builtin_amdgcn_readlane(v, at); };
            const int32_t local = number - units - (of(upto) - of(my_units));
            x.sequence = from + at;
            x.parts = of(parts);
            x.tile = BY_TILE ? local : local / x.parts;
            x.part = BY_TILE ? 0 : local - x.tile * x.parts;
            // (the latest tiles of a prompt see the most and are taken first)
            x.tile = of(mine.tiles) - 1 - x.tile;
            x.slot = slots + of(slots_upto) - of(my_slots) + x.tile * x.parts;
            x.first_token = of(mine.first);
            x.rows = of(mine.taken) * a.group;
            x.first_position = (int64_t)of(mine.length) - of(mine.count);
            const int32_t row = x.tile * a.tile_rows, last = min(row + a.tile_rows, x.rows) - 1;
            const int64_t p0 = x.first_position + a.by_group.divide(row), p1 = x.first_position + a.by_group.divide(last);
            x.low = (int32_t)max((int64_t)0, a.window ? p0 - a.window + 1 : 0) / kStep * kStep;
            x.high = (int32_t)max((int64_t)0, min(p1 + 1, (int64_t)a.c.capacity));
            const int32_t span = max(0, x.high - x.low);
            x.size = ((span + x.parts - 1) / x.parts + kStep - 1) / kStep * kStep;
            return true;
        }
        units += all;
        slots += __builtin_amdgcn_readlane(slots_upto, kWave - 1);
    }
    return false;
}

}  // namespace hbp
