// Host side of the paged 4-bit cache: argument checks and launches of the calls that lychee.h declares for it.
#include "lychee_context.h"
#include "lychee_host.h"
#include "lychee_paged.h"

#include <math.h>
#include <string.h>

using namespace lychee;

namespace {

int check_paged(const lychee_paged *p)
{
    if (p == nullptr) return LYCHEE_EINVAL;
    if (p->batch < 1 || p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_pages < 1 || p->max_pages < 1 || p->k < 1) return LYCHEE_EINVAL;
    if (p->n_q_heads % p->n_kv_heads != 0) return LYCHEE_EINVAL;
    if (p->head_dim != kHeadDim) return LYCHEE_EUNSUPPORTED;
    if (p->n_kv_heads > kMaxKvHeads || p->batch > kMaxBatch) return LYCHEE_EUNSUPPORTED;
    if (p->page_size != 16 && p->page_size != 32 && p->page_size != 64 && p->page_size != 128 && p->page_size != 256)
        return LYCHEE_EUNSUPPORTED;
    if (p->table_stride < p->max_pages || p->page_tiles < p->n_kv_heads * (p->page_size / kTileTokens)) return LYCHEE_EINVAL;
    if ((int64_t)p->max_pages * p->page_size > kMaxContext) return LYCHEE_EUNSUPPORTED;
    if ((int64_t)p->n_pages * p->page_size > INT32_MAX || (int64_t)p->n_pages * p->page_tiles > kMaxTiles) return LYCHEE_EUNSUPPORTED;
    return LYCHEE_OK;
}

int check_heads(const lychee_paged *p, const uint8_t *mask, bool has_idx_in)
{
    for (int h = 0; h < p->n_q_heads; ++h) {
        if (mask[h] > 1) return LYCHEE_EINVAL;
        if (mask[h] == 0 && !has_idx_in) return LYCHEE_EINVAL;
    }
    return LYCHEE_OK;
}

struct Carved {
    size_t part_o, part_ml, total;
};
Carved carve(const lychee_paged &p)
{
    const int64_t heads = q4_slots(p.batch, 2 * p.n_kv_heads, kQ4MaxWg) * (p.n_q_heads / p.n_kv_heads);
    Carved c;
    c.part_o = 0;
    c.part_ml = (size_t)round_up(heads * kHeadDim * (int64_t)sizeof(float), 256);
    c.total = c.part_ml + (size_t)round_up(heads * 2 * (int64_t)sizeof(float), 256);
    return c;
}

uint32_t *arrived_word(lychee_ctx *ctx) { return reinterpret_cast<uint32_t *>(ctx->sync_dev + kSyncPages); }

}  // namespace

extern "C" {

int lychee_check_paged(const lychee_paged *paged, const uint8_t *head_type_mask, int has_idx_in)
{
    const int rc = check_paged(paged);
    if (rc != LYCHEE_OK || head_type_mask == nullptr) return rc;
    return check_heads(paged, head_type_mask, has_idx_in != 0);
}

size_t lychee_paged_workspace_bytes(const lychee_paged *paged)
{
    return check_paged(paged) == LYCHEE_OK ? carve(*paged).total : 0;
}

int lychee_release_pages(lychee_ctx *ctx, const lychee_paged *paged, const uint8_t *done_flags, const int32_t *lengths,
                         const int32_t *block_table, int32_t *free_pages, const int32_t *free_count, int32_t *lengths_out,
                         int32_t *free_count_out, void *hip_stream)
{
    if (ctx == nullptr) return LYCHEE_EINVAL;
    const int rc = check_paged(paged);
    if (rc != LYCHEE_OK) return rc;
    if (!done_flags || !lengths || !block_table || !free_pages || !free_count || !lengths_out || !free_count_out) return LYCHEE_EINVAL;
    if (!aligned(lengths, 4) || !aligned(block_table, 4) || !aligned(free_pages, 4) || !aligned(free_count, 4) ||
        !aligned(lengths_out, 4) || !aligned(free_count_out, 4))
        return LYCHEE_EINVAL;
    const OnDevice dev(ctx);
    if (!dev.ok) return LYCHEE_EHIP;
    const ReleaseArgs a{dims_of(*paged), done_flags, lengths, block_table, free_count, free_pages, lengths_out, free_count_out,
                        arrived_word(ctx)};
    return done(launch_release(a, static_cast<hipStream_t>(hip_stream)));
}

int lychee_plan_pages(lychee_ctx *ctx, const lychee_paged *paged, const int32_t *lengths, const int32_t *new_tokens,
                      int32_t *block_table, const int32_t *free_pages, const int32_t *free_count, int32_t *lengths_out,
                      int32_t *free_count_out, int32_t *slots, int32_t n_slots, int32_t *token_start, int32_t *status,
                      void *hip_stream)
{
    if (ctx == nullptr) return LYCHEE_EINVAL;
    const int rc = check_paged(paged);
    if (rc != LYCHEE_OK) return rc;
    if (!lengths || !new_tokens || !block_table || !free_pages || !free_count || !lengths_out || !free_count_out || !token_start ||
        !status || n_slots < 0 || (n_slots > 0 && !slots))
        return LYCHEE_EINVAL;
    if (!aligned(lengths, 4) || !aligned(new_tokens, 4) || !aligned(block_table, 4) || !aligned(free_pages, 4) ||
        !aligned(free_count, 4) || !aligned(lengths_out, 4) || !aligned(free_count_out, 4) || !aligned(slots, 4) ||
        !aligned(token_start, 4) || !aligned(status, 4))
        return LYCHEE_EINVAL;
    const OnDevice dev(ctx);
    if (!dev.ok) return LYCHEE_EHIP;
    const PlanArgs a{dims_of(*paged), lengths, new_tokens, free_pages, free_count, block_table, lengths_out, free_count_out, slots,
                     token_start, status, n_slots, arrived_word(ctx)};
    return done(launch_plan(a, static_cast<hipStream_t>(hip_stream)));
}

int lychee_q4_append(lychee_ctx *ctx, const lychee_paged *paged, const void *k_new, const void *v_new, int64_t stride_tok,
                     int64_t stride_head, const int32_t *slots, int32_t n_tokens, void *cache, void *hip_stream)
{
    if (ctx == nullptr) return LYCHEE_EINVAL;
    const int rc = check_paged(paged);
    if (rc != LYCHEE_OK) return rc;
    if (n_tokens < 0 || !cache || !aligned(cache, 128)) return LYCHEE_EINVAL;
    if (n_tokens == 0) return LYCHEE_OK;
    if (!k_new || !v_new || !slots || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(slots, 4)) return LYCHEE_EINVAL;
    if (stride_tok < 0 || stride_head < 0 || stride_tok % 8 || stride_head % 8) return LYCHEE_EINVAL;
    if (((int64_t)n_tokens + 15) / 16 * paged->n_kv_heads >= 1 << 24) return LYCHEE_EUNSUPPORTED;  // (a launch's threads are 32 bits)
    const OnDevice dev(ctx);
    if (!dev.ok) return LYCHEE_EHIP;
    const AppendArgs a{dims_of(*paged), static_cast<const uint16_t *>(k_new), static_cast<const uint16_t *>(v_new), stride_tok,
                       stride_head, slots, n_tokens, static_cast<uint8_t *>(cache)};
    return done(launch_append(a, static_cast<hipStream_t>(hip_stream)));
}

int lychee_q4_read(lychee_ctx *ctx, const lychee_paged *paged, const void *cache, const int32_t *block_table, const int32_t *first,
                   const int32_t *last, void *k_out, void *v_out, int64_t stride_batch, int64_t stride_head, int64_t stride_tok,
                   int32_t n_rows, void *hip_stream)
{
    if (ctx == nullptr) return LYCHEE_EINVAL;
    const int rc = check_paged(paged);
    if (rc != LYCHEE_OK) return rc;
    if (!cache || !block_table || !last || !k_out || !v_out || n_rows < 0) return LYCHEE_EINVAL;
    if (!aligned(cache, 128) || !aligned(block_table, 4) || !aligned(first, 4) || !aligned(last, 4) || !aligned(k_out, 16) ||
        !aligned(v_out, 16))
        return LYCHEE_EINVAL;
    if (stride_tok < kHeadDim || stride_head < 0 || stride_batch < 0 || stride_tok % 8 || stride_head % 8 || stride_batch % 8)
        return LYCHEE_EINVAL;
    if ((paged->n_kv_heads > 1 && stride_head == 0) || (paged->batch > 1 && stride_batch == 0)) return LYCHEE_EINVAL;
    if (n_rows == 0) return LYCHEE_OK;
    const OnDevice dev(ctx);
    if (!dev.ok) return LYCHEE_EHIP;
    ReadArgs a{dims_of(*paged), static_cast<const uint8_t *>(cache), block_table, first, last, static_cast<uint16_t *>(k_out),
               static_cast<uint16_t *>(v_out), stride_batch, stride_head, stride_tok, n_rows};
    if (a.n_rows > a.d.max_len) a.n_rows = a.d.max_len;  // (a request holds no more)
    return done(launch_read(a, static_cast<hipStream_t>(hip_stream)));
}

int lychee_q4_decode_attn(lychee_ctx *ctx, const lychee_paged *paged, const void *q, const void *cache, const int32_t *block_table,
                          const int32_t *lengths, const uint8_t *head_type_mask, const int32_t *idx_in, void *out, float *scores,
                          int64_t score_stride, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (ctx == nullptr) return LYCHEE_EINVAL;
    int rc = check_paged(paged);
    if (rc != LYCHEE_OK) return rc;
    const int G = paged->n_q_heads / paged->n_kv_heads;
    if (G > kQ4MaxGroup) return LYCHEE_EUNSUPPORTED;
    if (!q || !cache || !block_table || !lengths || !out) return LYCHEE_EINVAL;
    if (!aligned(q, 16) || !aligned(cache, 128) || !aligned(block_table, 4) || !aligned(lengths, 4) || !aligned(idx_in, 4) ||
        !aligned(out, 16) || !aligned(scores, 4))
        return LYCHEE_EINVAL;
    if (head_type_mask != nullptr && (rc = check_heads(paged, head_type_mask, idx_in != nullptr)) != LYCHEE_OK) return rc;
    const Carved w = carve(*paged);
    if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < w.total) return LYCHEE_EWORKSPACE;
    Q4AttnArgs a;
    memset(&a, 0, sizeof a);
    a.d = dims_of(*paged);
    if (scores != nullptr && score_stride < a.d.max_len) return LYCHEE_EINVAL;
    for (int g = 0; g < paged->n_kv_heads; ++g) {
        uint32_t bits = 0;
        for (int i = 0; i < G; ++i)
            if (head_type_mask == nullptr || head_type_mask[g * G + i]) bits |= 1u << i;
        a.rmask[g] = (uint16_t)bits;
        if (bits != 0) a.rhead[a.n_rseg++] = (uint8_t)g;
        if (bits != (1u << G) - 1u) a.ghead[a.n_gseg++] = (uint8_t)g;
    }
    const int64_t seg_blocks = (a.d.max_len + kQ4Block - 1) / kQ4Block;
    const int64_t set_blocks = ((paged->k < a.d.max_len ? paged->k : a.d.max_len) + kQ4Block - 1) / kQ4Block;
    const int64_t most = (int64_t)paged->batch * (a.n_rseg * seg_blocks + a.n_gseg * set_blocks);
    if (most >= INT32_MAX / 2) return LYCHEE_EUNSUPPORTED;
    // a pending select still reads this workspace
    if (ctx->pending.active && ctx->pending.workspace == workspace) return LYCHEE_EINVAL;
    const OnDevice dev(ctx);
    if (!dev.ok) return LYCHEE_EHIP;
    a.q = static_cast<const uint16_t *>(q);
    a.cache = static_cast<const uint8_t *>(cache);
    a.table = block_table;
    a.lengths = lengths;
    a.idx_in = idx_in;
    a.out = static_cast<uint16_t *>(out);
    a.scores = scores;
    a.score_stride = score_stride;
    a.part_o = reinterpret_cast<float *>(static_cast<char *>(workspace) + w.part_o);
    a.part_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) + w.part_ml);
    a.seg_count = reinterpret_cast<uint32_t *>(ctx->sync_dev + kSyncSeg);
    a.n_wg = ctx->n_cu * kQ4WgPerCu;
    if (a.n_wg > kQ4MaxWg) a.n_wg = kQ4MaxWg;
    // (a piece is four blocks at least, or a whole segment)
    const int64_t pieces = (int64_t)paged->batch * (a.n_rseg * ((seg_blocks + kWaves - 1) / kWaves) + a.n_gseg * ((set_blocks + kWaves - 1) / kWaves));
    if (a.n_wg > pieces) a.n_wg = (int32_t)pieces;
    a.scale = (float)(1.0 / sqrt((double)kHeadDim));
    a.scale_log2e = (float)(1.4426950408889634 / sqrt((double)kHeadDim));
    return done(launch_q4_attn(a, static_cast<hipStream_t>(hip_stream)));
}

int lychee_select_scores(lychee_ctx *ctx, const lychee_paged *paged, const float *scores, int64_t score_stride,
                         const int32_t *lengths, const uint8_t *head_type_mask, const int32_t *idx_in, int32_t *idx_out,
                         void *hip_stream)
{
    if (ctx == nullptr) return LYCHEE_EINVAL;
    int rc = check_paged(paged);
    if (rc != LYCHEE_OK) return rc;
    if (!scores || !lengths || !idx_out || !aligned(scores, 4) || !aligned(lengths, 4) || !aligned(idx_in, 4) || !aligned(idx_out, 4))
        return LYCHEE_EINVAL;
    if (idx_in == idx_out) return LYCHEE_EINVAL;
    SelectArgs a;
    memset(&a, 0, sizeof a);
    a.d = dims_of(*paged);
    if (score_stride < a.d.max_len) return LYCHEE_EINVAL;
    for (int g = 0; g < paged->n_kv_heads; ++g) {
        bool any = head_type_mask == nullptr;
        for (int i = 0; i < a.d.group && head_type_mask != nullptr; ++i) {
            if (head_type_mask[g * a.d.group + i] > 1) return LYCHEE_EINVAL;
            any |= head_type_mask[g * a.d.group + i] != 0;
        }
        if (any) a.selects |= 1ull << g;
        else if (idx_in == nullptr) return LYCHEE_EINVAL;
    }
    const OnDevice dev(ctx);
    if (!dev.ok) return LYCHEE_EHIP;
    a.scores = scores;
    a.score_stride = score_stride;
    a.lengths = lengths;
    a.idx_in = idx_in;
    a.idx_out = idx_out;
    return done(launch_select(a, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
