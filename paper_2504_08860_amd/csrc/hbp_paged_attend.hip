// Attention of new tokens over a paged cache: checks, how the work is divided, launches by type (hbp_paged_attention).
#include "hbp_paged_attend.h"

#include <algorithm>
#include <cmath>

namespace hbp {
namespace {

// How the work is divided, from what the host knows: sizes, not the sequences' lengths.
int plan(const hbp_paged_t *cache, int64_t tokens, int heads, int window, int64_t most_new, Attend *a, size_t *bytes)
{
    const int rc = check_paged(cache, &a->c);
    if (rc != HBP_OK) return rc;
    if (tokens < 0 || heads < 1 || heads % cache->kv_heads || window < 0 || most_new < 0) return HBP_ERR_INVALID_ARGUMENT;
    const int64_t group = heads / cache->kv_heads;
    if (heads > 65536 || tokens * group >= (int64_t(1) << 31) - 65536) return HBP_ERR_TOO_LARGE;
    *bytes = 0;
    if (tokens == 0 || cache->sequences == 0 || most_new == 0) return HBP_OK;
    most_new = std::min(most_new, tokens);
    a->tokens = (int32_t)tokens;
    a->heads = heads;
    a->group = (int32_t)group;
    a->most_new = (int32_t)most_new;
    a->window = window;
    a->by_group = Divider::of(group);
    // Rows of a tile.  16 or 32 by k_attend, whose wavefronts share the rows and not the positions: best where the cache's bytes bound it; more by k_attend_rows, whose wavefronts have 16 rows or 32,
    // and 32 where that leaves enough to do for the chip's 256 places, parts of 512 positions counted (4 x 60 tokens of 4 heads: 21.1 us, with 16 16.2; 512 tokens over 30000 305 and 396).
    const int64_t most_rows = most_new * group, span = window ? std::min<int64_t>(a->c.capacity, (int64_t)window + most_new) : a->c.capacity;
    const bool wide = cache->head_dim * type_bytes(cache->type) > 256, any_page = cache->page_size % 8 != 0;
    const bool plenty = (tokens * group / 256 + cache->sequences) * cache->kv_heads * ((span + 511) / 512) >= 256;
    a->tile_rows = most_rows <= 16 || any_page ? 16 : most_rows <= 32 && cache->type != HBP_F32 && !wide ? 32 : most_rows <= 128 || wide || !plenty ? 128 : 256;
    const int64_t rows = a->tile_rows;
    a->tiles = std::min(tokens * group / rows + cache->sequences, cache->sequences * ((most_new * group + rows - 1) / rows));
    a->least = rows <= 32 ? 4 * kStep : cache->type == HBP_F32 ? 512 : 256;   // (4 x 60 tokens of 32 heads over 1000 positions: 29.3 us, with 512 32.3; 7 x 37 in fp32 over ragged 3000 49.7 and 47.7)
    a->enough = rows > 32 ? 2048 : 512;
    a->whole = a->tiles * cache->kv_heads < 128 ? 512 : 1024;   // (16 x 8 tiles of 1000 positions in two parts 20.9 us, whole 17.6; 8 of them 13.2 and 16.8)
    a->places = (int32_t)std::max<int64_t>(1, (rows > 32 ? 256 : 512) / cache->kv_heads);
    a->aim = (int32_t)std::max<int64_t>(1, (rows > 32 ? 512 : 1024) / cache->kv_heads);
    // Parts of tiles that are split: each is of more than `length` positions, so that its parts are at most twice its positions by `length`, and in all twice `aim`.
    const int64_t most_span = window ? std::min<int64_t>(a->c.capacity, (int64_t)window + rows) : a->c.capacity, most_parts = most_span <= a->whole ? 1 : (most_span + a->least - 1) / a->least;
    a->slots = most_parts < 2 ? 0 : (int32_t)std::min<int64_t>(2 * a->aim + 2, a->tiles * most_parts);
    a->units = std::min(a->tiles + a->aim + 1, a->tiles * std::max<int64_t>(most_parts, 1));   // (each tile one more than its positions by a part's)
    *bytes = (size_t)a->slots * cache->kv_heads * rows * (cache->head_dim * sizeof(float) + sizeof(float2));
    return HBP_OK;
}

}  // namespace
}  // namespace hbp

extern "C" {

int hbp_paged_attention_workspace(const hbp_paged_t *cache, int64_t tokens, int heads, int window, int64_t most_new, size_t *bytes)
{
    hbp::Attend a{};
    size_t need = 0;
    const int rc = hbp::plan(cache, tokens, heads, window, most_new, &a, &need);
    if (rc != HBP_OK || !bytes) return rc != HBP_OK ? rc : HBP_ERR_INVALID_ARGUMENT;
    *bytes = need;
    return HBP_OK;
}

int hbp_paged_attention(const hbp_paged_t *cache, int64_t tokens, const void *q, int64_t ldq, int heads, void *out, int64_t ldo, float scale, float softcap,
                        int window, int64_t most_new, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace hbp;
    Attend a{};
    size_t need = 0;
    int rc = plan(cache, tokens, heads, window, most_new, &a, &need);
    if (rc != HBP_OK) return rc;
    constexpr float kPerLog2 = 1.4426950408889634f;
    // (both are multiplied by 1 / log 2 below, and a larger cap's reciprocal would be no normal number)
    if (!std::isfinite(scale * kPerLog2) || !(softcap >= 0 && softcap <= 1e30f) || (softcap > 0 && !std::isfinite(scale / softcap * 3.0f))) return HBP_ERR_INVALID_ARGUMENT;
    if (a.tokens == 0) return HBP_OK;
    const int64_t bytes = type_bytes(cache->type), row = (int64_t)heads * cache->head_dim;
    if (!q || !out || !aligned(q, bytes) || !aligned(out, bytes) || (tokens > 1 && (ldq < row || ldo < row))) return HBP_ERR_INVALID_ARGUMENT;
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return HBP_ERR_INVALID_ARGUMENT;
    rc = earlier_error();
    if (rc != HBP_OK) return rc;
    a.q = q; a.ldq = ldq; a.out = out; a.ldo = ldo;
    a.keep = scale == 0 ? 0u : 0xffffffffu;
    a.flip = scale < 0 ? (cache->type == HBP_F32 ? 0x80000000u : 0x80008000u) : 0u;
    a.per = scale == 0 ? 1.0f : std::fabs(scale) * kPerLog2;
    if (softcap > 0) {
        a.cap_in = std::fabs(scale) / softcap;
        a.cap_out = softcap * kPerLog2;
    }
    const int64_t places = (int64_t)a.slots * cache->kv_heads * a.tile_rows;
    a.partial = static_cast<float *>(workspace);
    a.partial_stats = reinterpret_cast<float2 *>(a.partial + places * cache->head_dim);
    hipStream_t st = (hipStream_t)stream;
    switch (cache->type) {
    case HBP_F32: return launch_attend_f32(a, st);
    case HBP_F16: return launch_attend_f16(a, st);
    default: return launch_attend_bf16(a, st);
    }
}

}  // extern "C"
