// Host side of attention over whole prompts: argument checks and launches of the calls that lychee.h declares for it.
#include "lychee_context.h"
#include "lychee_host.h"
#include "lychee_prompt.h"

#include <math.h>
#include <string.h>

using namespace lychee;

namespace {

constexpr int32_t kPromptSlots = 512;  // ranges that fill a device: two workgroups a compute unit
constexpr int64_t kMaxGrid = 1 << 24;  // workgroups of 256 threads, which are counted in 32 bits

int check_heads_of(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim)
{
    if (n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads != 0) return LYCHEE_EINVAL;
    if (head_dim != kHeadDim || n_kv_heads > kMaxKvHeads || n_q_heads / n_kv_heads > kPromptMaxGroup) return LYCHEE_EUNSUPPORTED;
    return LYCHEE_OK;
}

bool good_stride(int64_t s) { return s >= 0 && s % 8 == 0; }

// Tiles of a batch's query rows, or of its keys, of a KV head, and the ranges that they are shared out to.
struct Grid {
    int64_t tiles, ranges, room;  // (room: ranges that a workspace has partials for, those of every smaller call too)
};
int64_t ranges_of(int64_t blocks, int32_t smallest, int32_t n_kv_heads)  // what fills the device, no more than there are smallest ranges
{
    const int64_t most = blocks / smallest + 1, fill = kPromptSlots / n_kv_heads;
    return most < fill ? most : fill;
}
// Whether lengths are possible with which a launch would share its tiles out (lay_line): a longest request against the least that
// it and the others can have, of equal lengths and, in a cache, with no keys but their own.  (To find out on the device, and a merge
// with nothing to do, cost 3 us: 17 tokens over 300 4-bit keys take 12.2 under a table for 512, 15.5 for 1024 and more.)
bool may_share(int32_t batch, int32_t heads, int32_t n_tokens, int64_t max_len, bool packed)
{
    const float range = (float)heads / (float)(kPromptRows * kPromptSlots), own = 1.f / (2 * kPromptKeys);
    const auto weight = [&](float tokens, float of_each) { return tokens * range * (of_each * own + kPromptTileCost); };
    const auto shared = [&](float longest, float all) {
        return longest / kPromptKeys + 1 + kPromptTileCost > kPromptShareCost + kPromptShareSize * all;
    };
    const float n = (float)n_tokens;
    if (!packed) return shared((float)max_len, weight(n, n / (float)batch));
    if (batch == 1) return shared(n, weight(n, n));
    for (int i = 1; i <= 12; ++i) {  // (one that has more than three quarters of all tokens is not looked for)
        const float longest = n * (float)i / 16, others = n - longest;
        if (shared(longest, weight(longest, longest) + weight(others, others / (float)(batch - 1)))) return true;
    }
    return false;
}
Grid rows_grid(int32_t batch, int32_t n_kv_heads, int32_t group, int32_t n_tokens, int64_t max_len, bool packed)
{
    Grid w;
    w.tiles = (int64_t)n_tokens * group / kPromptRows + (batch < n_tokens ? batch : n_tokens);
    const int64_t longest = max_len / kPromptKeys + 1 + kPromptTileCost;
    w.room = longest > kPromptShareCost ? ranges_of(w.tiles * longest, kPromptMinRange, n_kv_heads) : 0;
    w.ranges = w.room > 0 && may_share(batch, n_kv_heads * group, n_tokens, max_len, packed) ? w.room : 0;
    return w;
}
Grid keys_grid(int32_t batch, int32_t n_kv_heads, int32_t group, int32_t n_tokens)
{
    Grid w;
    w.tiles = n_tokens / kPromptRows + (batch < n_tokens ? batch : n_tokens);
    const int64_t blocks = w.tiles * ((int64_t)n_tokens * group / kPromptKeys + 1);
    w.room = ranges_of(blocks, kPromptMinKeyRange, n_kv_heads);
    w.ranges = blocks <= kPromptOneRange ? 1 : w.room;
    return w;
}

// A forward call's partials; a backward call's statistics and the partials of one launch after the other.
struct CarvedPrompt {
    size_t part_ml, stat, part, total;
};
CarvedPrompt carve(const Grid &w, int32_t n_kv_heads, int64_t stats, int64_t key_ranges)
{
    CarvedPrompt c;
    const size_t tile = kPromptRows * kHeadDim * sizeof(float), ml = kPromptRows * 2 * sizeof(float);
    const size_t of_rows = (size_t)(w.room * 2 * n_kv_heads), of_keys = (size_t)(key_ranges * 2 * n_kv_heads);
    const size_t records = (size_t)kPromptSlots * kRecordWords * sizeof(int32_t);  // (first)
    c.part_ml = records + of_rows * tile;
    c.stat = records;
    c.part = c.stat + (size_t)round_up(stats * 2 * (int64_t)sizeof(float), 256);
    const size_t forward = c.part_ml + of_rows * ml, rows = stats > 0 ? of_rows * tile : 0, keys = of_keys * 2 * tile;
    c.total = c.part + (rows > keys ? rows : keys);
    if (c.total < forward) c.total = forward;
    return c;
}

int check_prompt(const lychee_prompt *p)
{
    if (p == nullptr) return LYCHEE_EINVAL;
    if (p->batch < 1 || p->n_tokens < 0 || p->max_len < 0) return LYCHEE_EINVAL;
    const int rc = check_heads_of(p->n_q_heads, p->n_kv_heads, p->head_dim);
    if (rc != LYCHEE_OK) return rc;
    if (!good_stride(p->q_stride_tok) || !good_stride(p->q_stride_head) || !good_stride(p->kv_stride_batch) ||
        !good_stride(p->kv_stride_head) || !good_stride(p->kv_stride_tok) || p->q_stride_tok < kHeadDim || p->kv_stride_tok < kHeadDim)
        return LYCHEE_EINVAL;
    if (p->batch > kMaxBatch || p->max_len > kMaxContext) return LYCHEE_EUNSUPPORTED;
    if (p->q_stride_tok > kPromptMaxStride || p->q_stride_head > kPromptMaxStride || p->kv_stride_tok > kPromptMaxStride)
        return LYCHEE_EUNSUPPORTED;
    const int32_t G = p->n_q_heads / p->n_kv_heads;
    if ((int64_t)p->n_tokens * G >= kPromptMaxRows) return LYCHEE_EUNSUPPORTED;
    if (rows_grid(p->batch, p->n_kv_heads, G, p->n_tokens, 0, false).tiles * p->n_kv_heads >= kMaxGrid) return LYCHEE_EUNSUPPORTED;
    return LYCHEE_OK;
}

// Whether two rows, of tokens `tok` and heads `head` elements apart, have an element in common.
bool rows_meet(int64_t n_tokens, int64_t tok, int64_t n_heads, int64_t head)
{
    if (n_tokens == 0) return false;
    if ((n_tokens > 1 && tok < kHeadDim) || (n_heads > 1 && head < kHeadDim)) return true;
    if (n_tokens == 1 || n_heads == 1 || head >= (n_tokens - 1) * tok + kHeadDim || tok >= (n_heads - 1) * head + kHeadDim) return false;
    for (int64_t h = 1; h < n_heads; ++h) {  // head h of a token against the other tokens' first heads
        const int64_t t = h * head / tok, over = h * head - t * tok;
        if ((t > 0 && t < n_tokens && over < kHeadDim) || (t + 1 < n_tokens && tok - over < kHeadDim)) return true;
    }
    return false;
}

// The sizes of a call over the paged cache, and the tiles of its rows.
int check_q4(const lychee_paged *paged, int32_t n_tokens, Grid *rows)
{
    int rc = lychee_check_paged(paged, nullptr, 1);
    if (rc != LYCHEE_OK) return rc;
    const lychee_paged &p = *paged;
    if (n_tokens < 0) return LYCHEE_EINVAL;
    if ((rc = check_heads_of(p.n_q_heads, p.n_kv_heads, p.head_dim)) != LYCHEE_OK) return rc;
    const int32_t G = p.n_q_heads / p.n_kv_heads;
    if ((int64_t)n_tokens * G >= kPromptMaxRows) return LYCHEE_EUNSUPPORTED;
    *rows = rows_grid(p.batch, p.n_kv_heads, G, n_tokens, (int64_t)p.max_pages * p.page_size, false);
    return rows->tiles * p.n_kv_heads >= kMaxGrid ? LYCHEE_EUNSUPPORTED : LYCHEE_OK;
}

// (for either kind of keys: the longer request that a batch may hold)
CarvedPrompt carve(const lychee_prompt &p)
{
    const int32_t G = p.n_q_heads / p.n_kv_heads;
    return carve(rows_grid(p.batch, p.n_kv_heads, G, p.n_tokens, p.max_len > p.n_tokens ? p.max_len : p.n_tokens, false), p.n_kv_heads,
                 (int64_t)p.n_tokens * p.n_q_heads, keys_grid(p.batch, p.n_kv_heads, G, p.n_tokens).room);
}

PromptRows rows_of(int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_tokens, int32_t max_len, int64_t q_tok, int64_t q_head,
                   const int32_t *start, const int32_t *lengths)
{
    PromptRows r;
    memset(&r, 0, sizeof r);
    r.start = start;
    r.lengths = lengths;
    r.batch = batch;
    r.n_kv_heads = n_kv_heads;
    r.group = n_q_heads / n_kv_heads;
    r.n_tokens = n_tokens;
    r.max_len = max_len;
    r.group_magic = r.group > 1 ? (uint32_t)(((1ull << 32) + (uint32_t)r.group - 1) / (uint32_t)r.group) : 0;
    r.q_tok = q_tok;
    r.q_head = q_head;
    return r;
}

int check_workspace(const void *workspace, size_t bytes, const CarvedPrompt &c)
{
    return workspace == nullptr || !aligned(workspace, 256) || bytes < c.total ? LYCHEE_EWORKSPACE : LYCHEE_OK;
}

// Whether the first `written` of these addresses (NULL: left out) are no other argument's.
template <size_t N>
bool apart(const void *const (&at)[N], size_t written)
{
    for (size_t i = 0; i < written; ++i)
        for (size_t j = i + 1; j < N; ++j)
            if (at[i] != nullptr && at[i] == at[j]) return false;
    return true;
}

// A pending select still reads its workspace.
bool still_read(const lychee_ctx *ctx, const void *workspace) { return ctx->pending.active && ctx->pending.workspace == workspace; }

void fill_split(PromptArgs &a, const Grid &w, const CarvedPrompt &c, void *workspace)
{
    a.records = static_cast<int32_t *>(workspace);
    a.part_o = reinterpret_cast<float *>(static_cast<char *>(workspace) + c.stat);
    a.part_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) + c.part_ml);
    a.n_ranges = (int32_t)w.ranges;
    a.n_tiles = (int32_t)w.tiles;
    a.one_range = w.ranges > 0 ? 1.0 / (double)w.ranges : 0.0;
    a.by_number = w.tiles < w.ranges;
    a.n_records = a.by_number ? a.n_tiles : a.n_ranges;
    // (512 workgroups at least, two a compute unit, if 16 groups of dimensions are enough for that)
    a.merge_split = 1;
    while (a.merge_split < 16 && a.n_records * a.r.n_kv_heads * kWaves * a.merge_split < 512) a.merge_split *= 2;
    a.scale_log2e = (float)(1.4426950408889634 / sqrt((double)kHeadDim));
}

}  // namespace

extern "C" {

int lychee_check_prompt(const lychee_prompt *prompt) { return check_prompt(prompt); }

size_t lychee_prompt_workspace_bytes(const lychee_prompt *prompt) { return check_prompt(prompt) == LYCHEE_OK ? carve(*prompt).total : 0; }

int lychee_prompt_attn(lychee_ctx *ctx, const lychee_prompt *prompt, const void *q, const void *k, const void *v,
                       const int32_t *token_start, const int32_t *lengths, void *out, float *lse, void *workspace,
                       size_t workspace_bytes, void *hip_stream)
{
    if (ctx == nullptr) return LYCHEE_EINVAL;
    int rc = check_prompt(prompt);
    if (rc != LYCHEE_OK) return rc;
    const lychee_prompt &p = *prompt;
    if (!token_start || !aligned(token_start, 4) || !aligned(lengths, 4) || !aligned(lse, 4)) return LYCHEE_EINVAL;
    const CarvedPrompt c = carve(p);
    if ((rc = check_workspace(workspace, workspace_bytes, c)) != LYCHEE_OK) return rc;
    if (p.n_tokens == 0) return LYCHEE_OK;
    if (!q || !k || !v || !out || !aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16)) return LYCHEE_EINVAL;
    if (!apart({out, lse, workspace, q, k, v, token_start, lengths}, 3)) return LYCHEE_EINVAL;
    if (still_read(ctx, workspace)) return LYCHEE_EINVAL;
    const OnDevice dev(ctx);
    if (!dev.ok) return LYCHEE_EHIP;
    PromptArgs a;
    memset(&a, 0, sizeof a);
    a.r = rows_of(p.batch, p.n_q_heads, p.n_kv_heads, p.n_tokens, p.max_len, p.q_stride_tok, p.q_stride_head, token_start, lengths);
    a.q = static_cast<const uint16_t *>(q);
    a.k = static_cast<const uint16_t *>(k);
    a.v = static_cast<const uint16_t *>(v);
    a.kv_batch = p.kv_stride_batch;
    a.kv_head = p.kv_stride_head;
    a.kv_tok = p.kv_stride_tok;
    a.out = static_cast<uint16_t *>(out);
    a.lse = lse;
    fill_split(a, rows_grid(p.batch, p.n_kv_heads, a.r.group, p.n_tokens, lengths ? p.max_len : p.n_tokens, !lengths), c, workspace);
    return done(launch_prompt(a, static_cast<hipStream_t>(hip_stream)));
}

int lychee_prompt_attn_backward(lychee_ctx *ctx, const lychee_prompt *prompt, const void *d_out, const void *q, const void *k,
                                const void *v, const void *out, const float *lse, const int32_t *token_start, void *dq, void *dk, void *dv,
                                void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (ctx == nullptr) return LYCHEE_EINVAL;
    int rc = check_prompt(prompt);
    if (rc != LYCHEE_OK) return rc;
    const lychee_prompt &p = *prompt;
    if (!token_start || !aligned(token_start, 4) || !aligned(lse, 4)) return LYCHEE_EINVAL;
    // gradients of rows that meet would be written by several workgroups
    if (rows_meet(p.n_tokens, p.q_stride_tok, p.n_q_heads, p.q_stride_head) ||
        rows_meet(p.n_tokens, p.kv_stride_tok, p.n_kv_heads, p.kv_stride_head))
        return LYCHEE_EINVAL;
    const CarvedPrompt c = carve(p);
    if ((rc = check_workspace(workspace, workspace_bytes, c)) != LYCHEE_OK) return rc;
    if (p.n_tokens == 0) return LYCHEE_OK;
    if (!d_out || !q || !k || !v || !out || !lse || !dq || !dk || !dv) return LYCHEE_EINVAL;
    if (!aligned(d_out, 16) || !aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(dq, 16) ||
        !aligned(dk, 16) || !aligned(dv, 16))
        return LYCHEE_EINVAL;
    if (!apart({dq, dk, dv, workspace, d_out, q, k, v, out, lse, token_start}, 4)) return LYCHEE_EINVAL;
    if (still_read(ctx, workspace)) return LYCHEE_EINVAL;
    const OnDevice dev(ctx);
    if (!dev.ok) return LYCHEE_EHIP;
    PromptGradArgs a;
    memset(&a, 0, sizeof a);
    a.r = rows_of(p.batch, p.n_q_heads, p.n_kv_heads, p.n_tokens, p.max_len, p.q_stride_tok, p.q_stride_head, token_start, nullptr);
    a.g = static_cast<const uint16_t *>(d_out);
    a.q = static_cast<const uint16_t *>(q);
    a.k = static_cast<const uint16_t *>(k);
    a.v = static_cast<const uint16_t *>(v);
    a.out = static_cast<const uint16_t *>(out);
    a.lse = lse;
    a.kv_head = p.kv_stride_head;
    a.kv_tok = p.kv_stride_tok;
    a.dq = static_cast<uint16_t *>(dq);
    a.dk = static_cast<uint16_t *>(dk);
    a.dv = static_cast<uint16_t *>(dv);
    a.records = static_cast<int32_t *>(workspace);
    a.stat = reinterpret_cast<float *>(static_cast<char *>(workspace) + c.stat);
    a.scale = (float)(1.0 / sqrt((double)kHeadDim));
    a.scale_log2e = (float)(1.4426950408889634 / sqrt((double)kHeadDim));
    a.root = (float)sqrt((double)kHeadDim);
    const Grid rows = rows_grid(p.batch, p.n_kv_heads, a.r.group, p.n_tokens, p.n_tokens, true);
    const Grid keys = keys_grid(p.batch, p.n_kv_heads, a.r.group, p.n_tokens);
    a.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + c.part);
    a.n_row_ranges = (int32_t)rows.ranges;
    a.n_key_ranges = (int32_t)keys.ranges;
    a.n_row_tiles = (int32_t)rows.tiles;
    a.one_row_range = rows.ranges > 0 ? 1.0 / (double)rows.ranges : 0.0;
    a.one_key_range = 1.0 / (double)keys.ranges;
    a.rows_by_number = rows.tiles < rows.ranges;
    a.n_row_records = (int32_t)(a.rows_by_number ? rows.tiles : rows.ranges);
    a.keys_by_number = keys.tiles < keys.ranges;
    a.n_key_records = (int32_t)(a.keys_by_number ? keys.tiles : keys.ranges);
    return done(launch_prompt_grad(a, static_cast<hipStream_t>(hip_stream)));
}

size_t lychee_q4_prompt_workspace_bytes(const lychee_paged *paged, int32_t n_tokens)
{
    Grid w;
    return check_q4(paged, n_tokens, &w) == LYCHEE_OK ? carve(w, paged->n_kv_heads, 0, 0).total : 0;
}

int lychee_q4_prompt_attn(lychee_ctx *ctx, const lychee_paged *paged, const void *q, int64_t q_stride_tok, int64_t q_stride_head,
                          int32_t n_tokens, const void *cache, const int32_t *block_table, const int32_t *lengths,
                          const int32_t *token_start, void *out, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (ctx == nullptr) return LYCHEE_EINVAL;
    Grid w;
    int rc = check_q4(paged, n_tokens, &w);
    if (rc != LYCHEE_OK) return rc;
    const lychee_paged &p = *paged;
    if (q_stride_tok > kPromptMaxStride || q_stride_head > kPromptMaxStride) return LYCHEE_EUNSUPPORTED;
    if (!good_stride(q_stride_tok) || !good_stride(q_stride_head) || q_stride_tok < kHeadDim) return LYCHEE_EINVAL;
    if (!cache || !block_table || !lengths || !token_start || !aligned(cache, 128) || !aligned(block_table, 4) || !aligned(lengths, 4) ||
        !aligned(token_start, 4))
        return LYCHEE_EINVAL;
    const CarvedPrompt c = carve(w, p.n_kv_heads, 0, 0);
    if ((rc = check_workspace(workspace, workspace_bytes, c)) != LYCHEE_OK) return rc;
    if (n_tokens == 0) return LYCHEE_OK;
    if (!q || !out || !aligned(q, 16) || !aligned(out, 16)) return LYCHEE_EINVAL;
    if (!apart({out, workspace, q, cache, block_table, lengths, token_start}, 2)) return LYCHEE_EINVAL;
    if (still_read(ctx, workspace)) return LYCHEE_EINVAL;
    const OnDevice dev(ctx);
    if (!dev.ok) return LYCHEE_EHIP;
    PromptArgs a;
    memset(&a, 0, sizeof a);
    a.r = rows_of(p.batch, p.n_q_heads, p.n_kv_heads, n_tokens, p.max_pages * p.page_size, q_stride_tok, q_stride_head, token_start,
                  lengths);
    a.q = static_cast<const uint16_t *>(q);
    a.cache = static_cast<const uint8_t *>(cache);
    a.table = block_table;
    a.d = dims_of(p);
    a.out = static_cast<uint16_t *>(out);
    fill_split(a, w, c, workspace);
    return done(launch_prompt(a, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
