// What the operators of a batch of sequences share: which sequence a row is of, where a position lies in a paged cache.
#pragma once

#include "hbp_ops.h"

namespace hbp {

// Division of a number below 2^31 by a number from 1 to 2^31 - 1 that is fixed for a launch: with 2^(s-1) < d <= 2^s, m = ceil(2^(31+s) / d) is off by less than 2^s / d
// of its last place, so that n m / 2^(31+s) has the quotient's whole part.
struct Divider {
    uint32_t m, d;
    int32_t shift;
    static Divider of(int64_t d)
    {
        int s = 0;
        while ((int64_t(1) << s) < d) s++;
        const unsigned __int128 top = (unsigned __int128)1 << (31 + s);
        return Divider{(uint32_t)((top + (uint64_t)d - 1) / (uint64_t)d), (uint32_t)d, 31 + s};
    }
    __device__ __forceinline__ int32_t divide(int32_t n) const { return (int32_t)((uint64_t)(uint32_t)n * m >> shift); }
};

struct Paged {
    const void *keys, *values;
    const int32_t *table, *starts, *lengths;
    int64_t ldk, ldv, ldt;
    int32_t pages, sequences, table_width, kv_heads, page_size, head_dim;
    int32_t capacity;   // positions that a row of the table has pages for
    Divider by_page;
};

// The sequence of a row: how many sequences end at it or before it.  By a whole wavefront (64 ends at a time); `sequences` where it is of none.
__device__ __forceinline__ int32_t sequence_of(const int32_t *starts, int32_t sequences, int32_t row)
{
    const int lane = threadIdx.x % kWave;
    int32_t low = 0, high = sequences;   // the answer is in low..high
    while (low < high) {
        const int32_t step = (high - low + kWave - 1) / kWave;
        const int64_t at = (int64_t)low + (int64_t)(lane + 1) * step - 1;   // (the last one of each lane's share)
        const bool ended = at < high && starts[at + 1] <= row;
        const int32_t shares = __popcll(__ballot(ended));
        low = (int32_t)min((int64_t)low + (int64_t)shares * step, (int64_t)high);
        high = min(high, low + step - 1);
    }
    return low;
}

inline int check_paged(const hbp_paged_t *c, Paged *out)
{
    if (!c || !is_type(c->type) || c->kv_heads < 1 || c->page_size < 1 || c->pages < 1 || c->sequences < 0 || c->table_width < 1) return HBP_ERR_INVALID_ARGUMENT;
    if (c->head_dim < 8 || c->head_dim % 8 || c->head_dim > 256) return HBP_ERR_INVALID_ARGUMENT;
    if (c->page_size > 65536 || c->kv_heads > 65536 || c->pages >= (int64_t(1) << 31) || c->pages * c->page_size >= (int64_t(1) << 31) ||
        c->sequences > (int64_t(1) << 24) || c->table_width >= (int64_t(1) << 31)) return HBP_ERR_TOO_LARGE;
    const int64_t page = (int64_t)c->kv_heads * c->page_size * c->head_dim;
    if (c->ldk < page || c->ldv < page || c->ldk % 8 || c->ldv % 8 || (c->sequences > 1 && c->ldt < c->table_width)) return HBP_ERR_INVALID_ARGUMENT;
    if (!c->keys || !c->values || !aligned(c->keys, 16) || !aligned(c->values, 16)) return HBP_ERR_INVALID_ARGUMENT;
    if (c->sequences && (!c->table || !c->lengths)) return HBP_ERR_INVALID_ARGUMENT;
    if (!c->starts || !aligned(c->table, 4) || !aligned(c->starts, 4) || !aligned(c->lengths, 4)) return HBP_ERR_INVALID_ARGUMENT;
    const int64_t capacity = c->table_width * c->page_size, most = (int64_t(1) << 31) - 65537;
    *out = Paged{c->keys, c->values, c->table, c->starts, c->lengths, c->ldk, c->ldv, c->ldt, (int32_t)c->pages, (int32_t)c->sequences, (int32_t)c->table_width,
                 c->kv_heads, c->page_size, c->head_dim, (int32_t)(capacity < most ? capacity : most), Divider::of(c->page_size)};
    return HBP_OK;
}

}  // namespace hbp
