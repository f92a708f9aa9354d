// What the host side and the kernels of attention over whole prompts share: the kernels' arguments, the sizes of
// their launches.
#pragma once

#include "lychee_paged.h"

namespace lychee {

constexpr int kPromptMaxGroup = 16;
constexpr int kPromptRows = 128;          // query rows of a tile, a row being a (token, query head of the KV head)
constexpr int kPromptKeys = 64;           // keys a workgroup takes at a time
// Blocks in a range of row tiles, at least (17 rows over 2500 keys: 12.6 us with 2, 14.0 with 3, 14.9 with 4; over 6000: 18.1, 16.6, 16.5),
// and of key tiles.
constexpr int kPromptMinRange = 3;
constexpr int kPromptMinKeyRange = 2;
// Blocks of all key tiles (keys_grid counts them) that are one range, which needs no merge; more take a workgroup longer than ranges and
// their merge.  A backward call of 8 heads, 2 KV heads, in one range and in ranges: 32 tokens (3 blocks) 17.5 and 19.5 us, 48 (4) 20.5
// and 21.9, 64 (5) 23.3 and 22.1, 80 (6) 26.5 and 22.7, 96 (7) 30.3 and 24.0; of 64 heads, 16 KV heads, the same to 0.3 us.  (Three
// requests of 20 tokens, 8 heads each, 3 blocks in as many tiles: 22.4 and 19.8.)
constexpr int kPromptOneRange = 4;
// Rows' tiles are shared out where the longest has kPromptShareCost blocks more than kPromptShareSize times a range's (lay_line).
constexpr int kPromptShareCost = 14;
constexpr float kPromptShareSize = 1.6f;
constexpr int kPromptTileCost = 3;        // blocks that a row tile takes besides its own
constexpr int kRecordWords = 8;           // of a tile that several ranges share
constexpr int64_t kPromptMaxRows = 1 << 28;  // query tokens times heads of a group (row numbers are divided with a multiplication)
constexpr int64_t kPromptMaxStride = 1 << 24;  // elements from a token's row to the next (offsets within 64 rows fit 32 bits)

// A batch of packed query rows.
struct PromptRows {
    const int32_t *start;    // [batch + 1]
    const int32_t *lengths;  // [batch] keys of a request, or nullptr: as many as it has query tokens
    int32_t batch, n_kv_heads, group;
    int32_t n_tokens, max_len;
    uint32_t group_magic;    // ceil(2^32 / group): r / group = umulhi(r, magic) for group > 1 and r < kPromptMaxRows
    int64_t q_tok, q_head;   // strides of q, elements
};

struct PromptArgs {
    PromptRows r;
    const uint16_t *q, *k, *v;
    int64_t kv_batch, kv_head, kv_tok;  // strides of k and v; kv_batch counts where there are lengths
    const uint8_t *cache;               // the paged cache, or nullptr
    const int32_t *table;
    PagedDims d;
    uint16_t *out;      // [n_tokens][n_q_heads][128]
    float *lse;         // [n_q_heads][n_tokens] or nullptr
    float *part_o;      // [range][2][KV head][wavefront][16][64][4] un-normalised partial outputs, as registers and lanes hold them
    float *part_ml;     // [range][2][KV head][kPromptRows][2]       maximum (log2 units) and sum
    int32_t *records;   // [n_records][kRecordWords], by tile or by range
    int32_t n_records, by_number;
    double one_range;   // 1 / n_ranges
    int32_t n_ranges;   // 0: a workgroup a tile; else the workgroups that share a KV head's tiles
    int32_t n_tiles;    // of a KV head, at most
    int32_t merge_split;  // workgroups that share 32 rows of a tile in the merge
    float scale_log2e;
};

struct PromptGradArgs {
    PromptRows r;
    const uint16_t *g, *q, *k, *v, *out;
    const float *lse;
    int64_t kv_head, kv_tok;
    uint16_t *dq, *dk, *dv;  // strided like q, k and v
    float *stat;             // [2][n_q_heads][n_tokens] -lse sqrt(128), -(g . out): what the products of the second launch begin with
    float scale, scale_log2e, root;  // 1 / sqrt(128), log2(e) / sqrt(128), sqrt(128)
    float *part;             // partials of dq: [range][2][KV head][wavefront][16][64][4]; of dk and dv: twice as many in a wavefront
    int32_t *records;        // [n_records][kRecordWords], by tile or by range, of one launch after the other
    int32_t n_row_records, rows_by_number, n_key_records, keys_by_number;
    double one_row_range, one_key_range;
    int32_t n_row_ranges;    // 0: a workgroup a tile of rows; else those that share a KV head's
    int32_t n_key_ranges;    // workgroups that share a KV head's tiles of keys
    int32_t n_row_tiles;     // of a KV head, at most
};

hipError_t launch_prompt(const PromptArgs &a, hipStream_t stream);
hipError_t launch_prompt_grad(const PromptGradArgs &a, hipStream_t stream);

}  // namespace lychee
