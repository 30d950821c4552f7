// Attention of many rows over a paged cache (prompts): k_attend_rows, for pages of whole eights of positions.
#pragma once

#include "hbp_paged_attend_impl.h"

namespace hbp {
namespace {

// A workgroup of eight wavefronts takes 128 NQ rows, 16 NQ a wavefront, and walks through their positions in turns of 64 (heads of up to 64: 128, wider ones than 128: 32), which all of them read from LDS: keys and values come
// from the cache into registers two turns ahead, values are turned there (eight positions of one column become a lane's share of an operand), and both lie in LDS as operands of the matrix
// instruction, lane after lane, so that every read is one of 16 bytes a lane without conflicts.  Three buffers and one barrier a turn.  The scores of the next block of 32 positions are
// multiplied when this one's have become weights, or while they do.  Bound: the matrix cores (515 cycles a block of a wavefront with 2 x 16 rows of heads of 128) and the vector unit (some 80 instructions and 16 exponentials)
// in turn; 4 x 2048 bf16 tokens over up to 6000 positions, 32 heads of 128, 8 of keys: 735 us, 835 TFLOP/s, of which 28 are workgroups that find nothing to join, and the last turn of the chip, whose 256 places take 832 tiles of unequal length, leaves some 9 % of them idle;
// one prompt of 16384, whose tiles come out even: 2.26 ms, 975 TFLOP/s.  With 32 rows a wavefront an operand that
// has been read is multiplied twice; 64 would need accumulation registers, and copies from them (1356 us where this was 818); workgroups of four wavefronts, two on a compute unit, take 1.05 to 1.25 times as
// long; the two wavefronts of a SIMD in opposite phases, held there by barriers, 1.15 times.
constexpr int kRowThreads = 512;
template <typename T, int D> constexpr int row_turn() { return sizeof(T) == 4 ? (D == 64 ? 64 : 32) : 8192 / D; }
template <typename T, int D> constexpr int row_buffers() { return sizeof(T) == 4 && D > 128 ? 1 : 3; }   // (as LDS has room for)
template <typename T, int D> constexpr size_t row_lds() { return row_buffers<T, D>() * 2 * (size_t)row_turn<T, D>() * D * (sizeof(T) == 4 ? 6 : 2); }
template <typename T, int D, int NQ, bool WHOLE, bool FAR_CAP> __global__ __launch_bounds__(kRowThreads) void k_attend_rows(Attend a, int64_t first_unit)
{
    constexpr int kParts = sizeof(T) == 4 ? 3 : 1;             // of an operand, see Operand
    constexpr int kTurn = row_turn<T, D>(), kBuffers = row_buffers<T, D>(), kBlocks = kTurn / kStep, kEights = kTurn / 8;
    constexpr int kSteps = D / 32, kTiles = D / 16;
    constexpr int kOperand = 64 * 16 * kParts;                 // bytes of an operand of a wavefront
    constexpr int kKeyBytes = kBlocks * 2 * kSteps * kOperand, kBytes = 2 * kKeyBytes;   // (as many of values)
    constexpr int kChunks = D / 8, kKeyRows = kRowThreads / kChunks, kKeyLoads = kTurn / kKeyRows;   // keys: a thread loads a chunk of eight columns of neighbouring positions
    constexpr int kColumns = D * kEights / kRowThreads, kQuads = D / kColumns;                       // values: one or two columns of eight positions
    constexpr int kApart = 16 / (kTiles / kColumns), kSums = sizeof(T) == 4 && D < 256 ? 2 : 1;   // kSums: sums taken in turn
    constexpr bool kOrdered = sizeof(T) == 2 && (NQ == 2 || D == 256);   // weights first, then both products in an order that is given, see below (16 rows of 128: 4 x 60 tokens over 400 22.1 us, and 20.0 without)
    constexpr bool kLate = kOrdered && NQ == 2;                // where rows with far exponents are seen to, see below
    constexpr int kHead = kOrdered ? 2 : 0, kAtOnce = 8;       // key steps whose operands are read before weights are made; operands on their way
    static_assert(kKeyLoads >= 1 && 8 % kKeyLoads == 0 && kColumns >= 1 && kQuads * kEights == kRowThreads, "");
    extern __shared__ uint4 lds[];
    __shared__ int64_t keys_at[4][kEights], values_at[4][kEights];   // of four turns: where eight positions' rows begin, in values; odd: the cache does not hold them
    __shared__ uint32_t held_by[4];                                  // bits of the eights that it holds
    __shared__ int32_t odd_by[kBuffers];              // the last turn, and 1, in whose values there are infinities or NaN
    char *const base = reinterpret_cast<char *>(lds);
    const int lane = threadIdx.x % kWave, wave = one((int32_t)threadIdx.x / kWave), column = lane % 16, quarter = lane / 16;
    const int64_t number = first_unit + blockIdx.x;
    const int32_t unit_number = (int32_t)(number / a.c.kv_heads), kv_head = (int32_t)(number - (int64_t)unit_number * a.c.kv_heads);
    Unit x;
    if (!find_unit<false, kRowThreads>(a, unit_number, x)) return;
    const int32_t begin = x.low + x.part * x.size, end = min(begin + x.size, x.high);
    const int32_t *table = a.c.table + x.sequence * a.c.ldt;
    const int32_t dim = WHOLE ? D : a.c.head_dim;   // (WHOLE: loads of neighbouring rows have one address and offsets in their instructions, and nothing is behind the last column)
    const int32_t first_row = x.tile * a.tile_rows + wave * 16 * NQ;

    Operand<T> q[NQ][kSteps];
    int32_t low[NQ], count[NQ];
    int32_t all_low = 0, all_high = 0x7fffffff, some_low = 0x7fffffff, some_high = 0;   // positions that all rows of the wavefront see, and that some do
#pragma unroll
    for (int n = 0; n < NQ; n++) {
        const int32_t row = first_row + n * 16 + column;
        const bool is_row = row < x.rows;
        const int32_t token = a.by_group.divide(is_row ? row : 0), head = kv_head * a.group + (is_row ? row - token * a.group : 0);
        const T *from = static_cast<const T *>(a.q) + (int64_t)(x.first_token + token) * a.ldq + (int64_t)head * dim;
#pragma unroll
        for (int k = 0; k < kSteps; k++) {
            const int32_t at = 32 * k + 8 * quarter;
            Eight<T> v;
            v.clear();
            if (is_row && at < dim) v.load(from + at);
#pragma unroll
            for (int i = 0; i < Eight<T>::kWords; i++) v.w[i] = (v.w[i] & a.keep) ^ a.flip;
            q[n][k] = Operand<T>::of(v.w);
        }
        const int64_t position = x.first_position + token;
        low[n] = (int32_t)max((int64_t)0, a.window ? position - a.window + 1 : 0);
        const int32_t high = (int32_t)max((int64_t)0, min(position + 1, (int64_t)end));
        count[n] = is_row ? max(0, high - low[n]) : 0;
        if (is_row) {
            all_low = max(all_low, low[n]);
            all_high = min(all_high, high);
            if (count[n]) {
                some_low = min(some_low, low[n]);
                some_high = max(some_high, high);
            }
        }
    }
    auto least = [](int32_t p, int32_t q) { return min(p, q); };
    auto most = [](int32_t p, int32_t q) { return max(p, q); };
    all_low = one(wave_reduce(all_low, most));
    all_high = one(wave_reduce(all_high, least));
    some_low = one(wave_reduce(some_low, least));
    some_high = one(wave_reduce(some_high, most));
    // what the tile's rows see at all, and what all of them do
    const int32_t last_row = min((x.tile + 1) * a.tile_rows, x.rows) - 1;
    const int64_t p0 = x.first_position + a.by_group.divide(x.tile * a.tile_rows), p1 = x.first_position + a.by_group.divide(last_row);
    const int32_t tile_low = (int32_t)max((int64_t)x.low, a.window ? p0 - a.window + 1 : 0);
    const int64_t tile_all_low = a.window ? p1 - a.window + 1 : 0, tile_all_high = p0 + 1;

    const float per = a.cap_out != 0.0f ? 1.0f : a.per;   // (of what the cap has made of scores)
    float m[NQ], l[NQ];
    float4_t o[NQ][kTiles];
    int32_t far = 0;   // whether some row's largest exponent is far from 0 (the same in all lanes)
#pragma unroll
    for (int n = 0; n < NQ; n++) {
        m[n] = kLowest;
        l[n] = 0.0f;
#pragma unroll
        for (int j = 0; j < kTiles; j++) o[n][j] = float4_t{0, 0, 0, 0};
    }

    // A turn's keys and values on their way: loaded into registers, then put into LDS as operands.
    Piece<T, 8> kf[kKeyLoads];
    Piece<T, kColumns> vf[8];
    const int key_chunk = threadIdx.x % kChunks, key_row = threadIdx.x / kChunks * kKeyLoads;   // positions key_row ..
    const int quad = threadIdx.x % kQuads, eight = threadIdx.x / kQuads;
    // Where a turn's rows are is looked up once for each eight positions, by a thread of the first wavefront, two turns before they are loaded: the table's entry in one turn, the addresses in the next.
    const int32_t last_eight = (end - 1) / 8 * 8;
    int32_t entry = 0, entry_position = 0;
    auto look_up = [&](int32_t turn, int i) {   // (of positions moved back before the end: what is read there has no weight)
        entry_position = min(turn + 8 * i, last_eight);
        entry = table[a.c.by_page.divide(entry_position)];
    };
    auto tell = [&](int which, int i) {
        const bool held = entry >= 0 && entry < a.c.pages;
        const int64_t page = held ? entry : 0, row = (int64_t)kv_head * a.c.page_size * dim + (entry_position - a.c.by_page.divide(entry_position) * a.c.page_size) * dim;
        keys_at[which][i] = (page * a.c.ldk + row) | !held;   // (rows are of whole eights of values)
        values_at[which][i] = (page * a.c.ldv + row) | !held;
        return held;
    };
    bool held_next = true;
    const int32_t key_offset = key_row % 8 * dim + (8 * key_chunk < dim ? 8 * key_chunk : 0), value_offset = kColumns * quad < dim ? kColumns * quad : 0;
    auto load = [&](int turn_number) {
        const int64_t key_at = keys_at[turn_number % 4][key_row / 8], value_at = values_at[turn_number % 4][eight];
        held_next = !(value_at & 1);
        const T *keys = static_cast<const T *>(a.c.keys) + (key_at & ~(int64_t)1) + key_offset;
        const T *values = static_cast<const T *>(a.c.values) + (value_at & ~(int64_t)1) + value_offset;
#pragma unroll
        for (int i = 0; i < kKeyLoads; i++) kf[i].load(keys + i * dim);
#pragma unroll
        for (int i = 0; i < 8; i++) vf[i].load(values + i * dim);
    };
    auto look_ahead = [&](int turn_number) {   // in turn `turn_number`
        if (wave == 0) {
            bool held = true;
            if (lane < kEights) {
                held = tell((turn_number + 3) % 4, lane);
                look_up(begin + (turn_number + 4) * kTurn, lane);
            }
            const uint64_t bits = __ballot(held);
            if (lane == 0) held_by[(turn_number + 3) % 4] = (uint32_t)bits;
        }
    };
    // row r of half h of a block is its position 8 (r / 4) + 4 h + r % 4; a row's place among 16 changes with the chunk of columns, so that neither side meets a bank twice
    auto put = [&](int32_t turn, int which) {
        char *const keys = base + which * kBytes, *const values = keys + kKeyBytes;
        const bool held = held_next;
        const uint32_t there = WHOLE || 8 * key_chunk < dim ? 0xffffffffu : 0u;
        auto store = [](char *to, const Operand<T> &v) {
            const uint4_t *parts = reinterpret_cast<const uint4_t *>(&v);
#pragma unroll
            for (int k = 0; k < kParts; k++) *reinterpret_cast<uint4_t *>(to + k * 64 * 16) = parts[k];
        };
#pragma unroll
        for (int i = 0; i < kKeyLoads; i++) {
            const int position = key_row + i, block = position / kStep, h = position / 4 % 2, r = position / 8 % 4 * 4 + position % 4;
            const int operand = (block * 2 + h) * kSteps + key_chunk / 4;
#pragma unroll
            for (int w = 0; w < Piece<T, 8>::kWords; w++) kf[i].w[w] &= there;
            store(keys + operand * kOperand + (key_chunk % 4 * 16 + (r ^ (key_chunk % 16))) * 16, Operand<T>::of(kf[i].w));
        }
        // Values that no row sees must not be there at all, not even with a weight of 0; infinities and NaN are taken out where only some rows see them (in fp32 everywhere: parts of an
        // infinity make NaN), and added for those rows
        const bool edge = turn < tile_all_low || (int64_t)turn + kTurn > tile_all_high || turn + kTurn > end;   // (the same in all threads)
        if (edge || !held)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int32_t position = turn + 8 * eight + i;
                const uint32_t seen = held && position >= tile_low && position < end ? 0xffffffffu : 0u;
#pragma unroll
                for (int w = 0; w < Piece<T, kColumns>::kWords; w++) vf[i].w[w] &= seen;
            }
        if (edge || !held || sizeof(T) == 4) {
            uint32_t largest = 0;
#pragma unroll
            for (int i = 0; i < 8; i++) {
#pragma unroll
                for (int w = 0; w < Piece<T, kColumns>::kWords; w++) {
                    if constexpr (sizeof(T) == 4) largest = max(largest, vf[i].w[w] & 0x7fffffffu);
                    else largest = largest_halves(largest, vf[i].w[w] & 0x7fff7fffu);
                }
            }
            if ((edge || sizeof(T) == 4) && has_odd<T>(largest)) {
                odd_by[which] = turn + 1;   // (every thread that finds one says the same)
#pragma unroll
                for (int i = 0; i < 8; i++)
#pragma unroll
                    for (int w = 0; w < Piece<T, kColumns>::kWords; w++) vf[i].w[w] = without_odd<T>(vf[i].w[w]);
            }
        }
        // column c is row c / kTiles of tile c % kTiles
#pragma unroll
        for (int i = 0; i < kColumns; i++) {
            uint32_t w[sizeof(T) * 2];
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int k = 0; k < 8; k++) w[k] = vf[k].w[i];
            } else {
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const uint32_t one = vf[2 * k].w[i / 2], two = vf[2 * k + 1].w[i / 2];
                    w[k] = i & 1 ? high_halves(one, two) : low_halves(one, two);
                }
            }
            const int at = kColumns * quad + i, r = at / kTiles, j = at % kTiles;
            const int operand = eight / 4 * kTiles + j;
            store(values + operand * kOperand + (eight % 4 * 16 + (r ^ (j / kColumns * kApart))) * 16, Operand<T>::of(w));
        }
    };
    // what has been written to LDS is there for all; loads from the cache stay on their way
    auto barrier = [&] {
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    auto operand_at = [](const char *from) {
        Operand<T> v;
        uint4_t *parts = reinterpret_cast<uint4_t *>(&v);
#pragma unroll
        for (int k = 0; k < kParts; k++) parts[k] = *reinterpret_cast<const uint4_t *>(from + k * 64 * 16);
        return v;
    };
    auto key_at = [&](int which, int b, int k, int h) {
        return operand_at(base + which * kBytes + ((b * 2 + h) * kSteps + k) * kOperand + (quarter * 16 + (column ^ ((4 * k + quarter) % 16))) * 16);
    };
    Operand<T> head[kHead ? 2 * kHead : 1];
    auto read_head = [&](int which, int b) {
#pragma unroll
        for (int i = 0; i < 2 * kHead; i++) head[i] = key_at(which, b, i / 2, i % 2);
    };
    auto scores = [&](float4_t (&s)[NQ][2], int which, int b) {   // (after read_head)
#pragma unroll
        for (int n = 0; n < NQ; n++) s[n][0] = s[n][1] = float4_t{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < kSteps; k++) {
            Operand<T> key[2];
#pragma unroll
            for (int h = 0; h < 2; h++) key[h] = k < kHead ? head[k < kHead ? 2 * k + h : 0] : key_at(which, b, k, h);
#pragma unroll
            for (int product = 0; product < kProducts<T>; product++)
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int n = 0; n < NQ; n++) s[n][h] = multiply(key[h], q[n][k], s[n][h], product);
        }
    };

    if (threadIdx.x < kBuffers) odd_by[threadIdx.x] = 0;
    if (begin < end) {
        const int eights = 3 * kEights;
        for (int i = threadIdx.x; i < eights; i += kRowThreads) {
            look_up(begin, i);
            tell(i / kEights, i % kEights);
        }
        __syncthreads();
        if (wave == 0) {
            if (lane < 3) {
                uint32_t bits = 0;
                for (int i = 0; i < kEights; i++) bits |= (uint32_t)!(values_at[lane][i] & 1) << i;
                held_by[lane] = bits;
            }
            if (lane < kEights) look_up(begin + 3 * kTurn, lane);
        }
        load(0);
        if constexpr (kBuffers > 1) {
            put(begin, 0);
            load(1);
            barrier();
        }
        float4_t s[NQ][2];
        bool ready = false;    // s has the scores of the turn's first block
        int which = 0, turn_number = 0;
        for (int32_t turn = begin; turn < end; turn += kTurn, turn_number++) {
            const int following = kBuffers == 1 || which == 2 ? 0 : which + 1;
            if constexpr (kBuffers == 1) {
                __syncthreads();   // (nobody reads the turn before this one's operands any more)
                put(turn, 0);
                load(turn_number + 1);
                look_ahead(turn_number);
                barrier();
            }
            const bool active = turn < some_high && turn + kTurn > some_low;   // (the same in all lanes)
            if (active && (!ready || kBuffers == 1)) {
                read_head(which, 0);
                scores(s, which, 0);
            }
            ready = active;
            const uint32_t held = one(held_by[turn_number % 4]);
            const bool odd = one(odd_by[which]) == turn + 1;
#pragma unroll
            for (int b = 0; b < kBlocks; b++) {
                if (kBuffers > 1 && b == (kOrdered ? 0 : kBlocks - 1)) {
                    if (turn + kTurn < end) put(turn + kTurn, following);
                    load(turn_number + 2);
                    look_ahead(turn_number);
                }
                const int32_t block = turn + b * kStep;
                float less[NQ];
                if (active) {
                    if constexpr (sizeof(T) == 4)
#pragma unroll
                        for (int n = 0; n < NQ; n++) {
                            float e[8];
#pragma unroll
                            for (int i = 0; i < 8; i++) e[i] = s[n][i / 4][i % 4];
                            by_definition(a, x, table, kv_head, first_row + n * 16 + column, block, low[n], count[n], held >> (4 * b + quarter) & 1 ? 0xffu : 0u, e);
#pragma unroll
                            for (int i = 0; i < 8; i++) s[n][i / 4][i % 4] = e[i];
                        }
                    if (a.cap_out != 0.0f) {
#pragma unroll
                        for (int n = 0; n < NQ; n++) {
                            if constexpr (FAR_CAP) {
                                float e[8];
#pragma unroll
                                for (int i = 0; i < 8; i++) e[i] = s[n][i / 4][i % 4];
                                far_capped(a, e);
#pragma unroll
                                for (int i = 0; i < 8; i++) s[n][i / 4][i % 4] = e[i];
                            } else {
#pragma unroll
                                for (int i = 0; i < 8; i++) s[n][i / 4][i % 4] = capped<T>(a, s[n][i / 4][i % 4]);
                            }
                        }
                    }
                    if (block < all_low || block + kStep > all_high || (held >> (4 * b) & 0xf) != 0xf) {
#pragma unroll
                        for (int n = 0; n < NQ; n++)
#pragma unroll
                            for (int i = 0; i < 8; i++) {
                                const bool sees = (uint32_t)(block + 8 * quarter + i - low[n]) < (uint32_t)count[n] && (held >> (4 * b + quarter) & 1);
                                if (!sees) s[n][i / 4][i % 4] = -INFINITY;
                            }
                    }
                    float top[NQ];
                    bool larger = false;
#pragma unroll
                    for (int n = 0; n < NQ; n++) {
                        top[n] = s[n][0][0];
#pragma unroll
                        for (int i = 1; i < 8; i++) top[n] = fmaxf(top[n], s[n][i / 4][i % 4]);
                        top[n] *= per;
                        larger |= top[n] - m[n] > kSlack<T>;
                    }
                    if (__ballot(larger) != 0) {   // (see k_attend)
                        far = 0;
#pragma unroll
                        for (int n = 0; n < NQ; n++) {
                            const float to = over_quarters(fmaxf(top[n] - kUp<T>, m[n]), [](float p, float q) { return fmaxf(p, q); });
                            const float f = __builtin_amdgcn_exp2f(m[n] - to);
                            m[n] = to;
                            far |= __ballot(fabsf(to) >= kFarExponent && to > kLowest) != 0;
                            l[n] *= f;
#pragma unroll
                            for (int j = 0; j < kTiles; j++)
#pragma unroll
                                for (int i = 0; i < 4; i++) o[n][j][i] *= f;
                        }
                    }
                    // (far rows' scores are changed here, or their weights below: with 2 x 16 rows of 16 bits 812 us and 735, 4 x 2048 tokens; with heads of 256 873 and 889, fp32 prompts 224 and 232)
                    if constexpr (!kLate) {
#pragma unroll
                        for (int n = 0; n < NQ; n++) less[n] = m[n];
                        if (one(far))
#pragma unroll
                            for (int n = 0; n < NQ; n++) {
                                float e[8];
#pragma unroll
                                for (int i = 0; i < 8; i++) e[i] = s[n][i / 4][i % 4];
                                far_scores(e, m[n], per, less[n]);
#pragma unroll
                                for (int i = 0; i < 8; i++) s[n][i / 4][i % 4] = e[i];
                            }
                    }
                }
                if (kBuffers > 1 && b == kBlocks - 1) barrier();   // (the next turn's operands are in LDS; their buffer was read last in the turn before this one)
                if (active) {
                    const int next_which = b == kBlocks - 1 ? following : which, next_block = b == kBlocks - 1 ? 0 : b + 1;
                    if constexpr (kOrdered) {
                        read_head(next_which, next_block);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    Operand<T> weights[NQ];
                    float p[NQ][8];
#pragma unroll
                    for (int n = 0; n < NQ; n++)
#pragma unroll
                        for (int i = 0; i < 8; i++) p[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i / 4][i % 4], per, -(kLate ? m[n] : less[n])));
                    if constexpr (kLate)
                        if (one(far))
#pragma unroll
                            for (int n = 0; n < NQ; n++) {
                                float e[8];
#pragma unroll
                                for (int i = 0; i < 8; i++) e[i] = s[n][i / 4][i % 4];
                                far_weights(p[n], e, m[n], per);
                            }
#pragma unroll
                    for (int n = 0; n < NQ; n++) {
#pragma unroll
                        for (int i = 0; i < 8; i++) l[n] += p[n][i];
                        weights[n] = Operand<T>::of(p[n]);
                    }
                    if constexpr (kOrdered) __builtin_amdgcn_sched_barrier(0);
                    if (kBuffers > 1 || b < kBlocks - 1) scores(s, next_which, next_block);   // (behind the last turn of nothing, for nothing)
                    const char *const values = base + which * kBytes + kKeyBytes;
#pragma unroll
                    for (int j = 0; j < kTiles; j += kSums) {
                        Operand<T> value[kSums];
#pragma unroll
                        for (int c = 0; c < kSums; c++)
                            value[c] = operand_at(values + (b * kTiles + j + c) * kOperand + (quarter * 16 + (column ^ ((j + c) / kColumns * kApart))) * 16);
#pragma unroll
                        for (int product = 0; product < kProducts<T>; product++)
#pragma unroll
                            for (int c = 0; c < kSums; c++)
#pragma unroll
                                for (int n = 0; n < NQ; n++) o[n][j + c] = multiply(value[c], weights[n], o[n][j + c], product);
                    }
                    if constexpr (kOrdered) {
                        // kAtOnce operands on their way, two more for each two that have been multiplied (the compiler's own order has four, and waits for LDS: 747 us instead of 730, 895 instead of 861 with heads of 256)
                        constexpr int kReads = 2 * kSteps + kTiles;
                        __builtin_amdgcn_sched_group_barrier(0x100, kAtOnce - 2 * kHead, 0);
#pragma unroll
                        for (int i = 0; i < (kReads - kAtOnce) / 2; i++) {
                            __builtin_amdgcn_sched_group_barrier(0x008, 2 * NQ, 0);
                            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                        }
                        __builtin_amdgcn_sched_group_barrier(0x008, kAtOnce * NQ, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    if (odd)
                        add_odd<T, D, NQ>(a, table, kv_head, block, max(tile_low, block), min(end, block + kStep), weights, low, count, o);
                }
            }
            which = following;
        }
    }

#pragma unroll
    for (int n = 0; n < NQ; n++) {
        const float sum = over_quarters(l[n], [](float p, float q) { return p + q; });
        const int32_t row = first_row + n * 16 + column;
        if (row >= x.rows) continue;
        if (x.parts == 1) {
            const int32_t token = a.by_group.divide(row);
            T *to = static_cast<T *>(a.out) + (int64_t)(x.first_token + token) * a.ldo + (int64_t)(kv_head * a.group + row - token * a.group) * dim;
            const float inverse = 1.0f / sum;
#pragma unroll
            for (int k = 0; k < 4; k++) {
                // (columns kTiles (4 quarter + k) .. + kTiles - 1)
#pragma unroll
                for (int c = 0; c < kTiles; c += 4) {
                    const int32_t at = kTiles * (4 * quarter + k) + c;
                    struct __attribute__((packed, aligned(2))) { T v[4]; } four;
#pragma unroll
                    for (int i = 0; i < 4; i++) four.v[i] = from_f32<T>(sum == 0.0f ? 0.0f : o[n][c + i][k] * inverse);
                    if (at < dim) *reinterpret_cast<decltype(four) *>(to + at) = four;
                }
            }
        } else {
            const int64_t to = ((int64_t)(x.slot + x.part) * a.c.kv_heads + kv_head) * a.tile_rows + wave * 16 * NQ + n * 16 + column;
#pragma unroll
            for (int k = 0; k < 4; k++)
#pragma unroll
                for (int c = 0; c < kTiles; c += 4) {
                    const int32_t at = kTiles * (4 * quarter + k) + c;
                    if (at < dim) *reinterpret_cast<float4_t *>(a.partial + to * dim + at) = float4_t{o[n][c][k], o[n][c + 1][k], o[n][c + 2][k], o[n][c + 3][k]};
                }
            if (quarter == 0) a.partial_stats[to] = float2{m[n], sum};
        }
    }
}

template <typename T, int D, int NQ, bool WHOLE, bool FAR_CAP = false> int launch_rows(const Attend &a, hipStream_t st)
{
    constexpr int64_t kMost = int64_t(1) << 22;
    constexpr size_t kLds = row_lds<T, D>();
    auto kernel = k_attend_rows<T, D, NQ, WHOLE, FAR_CAP>;
    HBP_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds));
    const int64_t units = a.units * a.c.kv_heads;
    for (int64_t at = 0; at < units; at += kMost) {
        kernel<<<dim3((unsigned)std::min(units - at, kMost)), kRowThreads, kLds, st>>>(a, at);
        HBP_HIP(hipGetLastError());
    }
    return HBP_OK;
}

// Few rows by k_attend, many by k_attend_rows, as the tiles have been planned; then what was split.
template <typename T> int launch_attend(const Attend &a, hipStream_t st)
{
    const bool any = a.c.page_size % 8 != 0;
    auto by_rows = [&](auto d) -> int {
        constexpr int D = decltype(d)::value;
        if (any) return launch_units<T, D, 1, true>(a, st);
        if (a.tile_rows == 16) return launch_units<T, D, 1, false>(a, st);
        const bool whole = a.c.head_dim == D;
        // (large caps have kernels of their own: asked for in the loop, they make prompts without a cap take 1.01 to 1.04 times as long, with one of 30 1.07)
        if constexpr (sizeof(T) == 2)
            if (has_far_cap<T>(a) && a.tile_rows >= 128) {
                if constexpr (D * sizeof(T) < 512)
                    if (a.tile_rows == 256) return launch_rows<T, D, 2, false, true>(a, st);
                return launch_rows<T, D, 1, false, true>(a, st);
            }
        if (a.tile_rows == 128) return whole ? launch_rows<T, D, 1, true>(a, st) : launch_rows<T, D, 1, false>(a, st);
        if constexpr (D * sizeof(T) < 512)
            if (a.tile_rows == 256) return whole ? launch_rows<T, D, 2, true>(a, st) : launch_rows<T, D, 2, false>(a, st);
        if constexpr (D * sizeof(T) <= 256 && sizeof(T) == 2) return launch_units<T, D, 2, false>(a, st);
        return HBP_ERR_INVALID_ARGUMENT;   // (no such plan)
    };
    const int32_t dim = a.c.head_dim;
    const int rc = dim <= 64 ? by_rows(std::integral_constant<int, 64>()) : dim <= 128 ? by_rows(std::integral_constant<int, 128>()) : by_rows(std::integral_constant<int, 256>());
    if (rc != HBP_OK || a.slots == 0) return rc;
    constexpr int64_t kMost = int64_t(1) << 23;
    const int64_t joins = a.tiles * a.c.kv_heads * (a.tile_rows / 16);
    for (int64_t at = 0; at < joins; at += kMost) {
        const dim3 grid((unsigned)std::min(joins - at, kMost));
        auto join = [&](auto lanes) {
            if (a.tile_rows == 16) k_attend_join<T, decltype(lanes)::value, 1><<<grid, 256, 0, st>>>(a, at);
            else k_attend_join<T, decltype(lanes)::value, 4><<<grid, 256, 0, st>>>(a, at);
        };
        if (dim <= 64) join(std::integral_constant<int, 8>());
        else if (dim <= 128) join(std::integral_constant<int, 16>());
        else join(std::integral_constant<int, 32>());
        HBP_HIP(hipGetLastError());
    }
    return HBP_OK;
}

}  // namespace
}  // namespace hbp
