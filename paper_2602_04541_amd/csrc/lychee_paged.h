// What the host side and the kernels of the paged 4-bit cache share: its layout, the kernels' arguments, the
// sizes of their launches.
#pragma once

#include "lychee_internal.h"

namespace lychee {

constexpr int kTileTokens = 16;            // tokens of a tile: their rows, then one line of scales
constexpr int kTokenBytes = 128;           // a token's row: 64 bytes of key, 64 of value
constexpr int kTileBytes = kTileTokens * kTokenBytes + 128;
constexpr int kTileScales = kTileTokens * kTokenBytes;  // where the scales begin: [8][16] bytes
constexpr int kScaleMin = 127 - 125, kScaleMax = 127 + 125;  // scale bytes of finite groups
constexpr int kQ4Block = 64;               // tokens a wavefront takes at a time
constexpr int kQ4MaxGroup = 16;
constexpr int kSplits = 16;                // sizes of a piece that an attention launch weighs
constexpr int kPieceCost = 12;             // what a piece costs whatever its length, in blocks
constexpr int kCutCost = 160;              // and the weight of a cut where there are more pieces than workgroups (fitted)
constexpr int kQ4WgPerCu = 2;
constexpr int kQ4MaxWg = 512;              // upper bound of an attention launch's grid
constexpr int64_t kMaxTiles = 1 << 27;     // of a cache (292 GB)
constexpr int kMaxContext = 1 << 24;       // tokens a request can hold

// Sizes of a paged cache, as the kernels need them.
struct PagedDims {
    int32_t batch, n_kv_heads, group;
    int32_t n_pages, page_shift, max_len;  // max_len: tokens a request's table row holds
    int32_t table_stride, page_tiles, k;
};

struct ReleaseArgs {
    PagedDims d;
    const uint8_t *done;
    const int32_t *lengths, *table, *free_count;
    int32_t *free_pages, *lengths_out, *free_count_out;
    uint32_t *arrived;  // workgroups that have read the inputs; zero between launches
};

struct PlanArgs {
    PagedDims d;
    const int32_t *lengths, *new_tokens, *free_pages, *free_count;
    int32_t *table, *lengths_out, *free_count_out, *slots, *token_start, *status;
    int32_t n_slots;
    uint32_t *arrived;
};

struct AppendArgs {
    PagedDims d;
    const uint16_t *k_new, *v_new;
    int64_t stride_tok, stride_head;
    const int32_t *slots;
    int32_t n_tokens;
    uint8_t *cache;
};

struct ReadArgs {
    PagedDims d;
    const uint8_t *cache;
    const int32_t *table, *first, *last;
    uint16_t *k_out, *v_out;
    int64_t stride_b, stride_h, stride_t;
    int32_t n_rows;
};

struct Q4AttnArgs {
    PagedDims d;
    const uint16_t *q;
    const uint8_t *cache;
    const int32_t *table, *lengths, *idx_in;
    uint16_t *out;
    float *scores;        // or nullptr
    int64_t score_stride;
    float *part_o;        // [slot][group][128] un-normalised partial outputs
    float *part_ml;       // [slot][group][2]   running maximum (log2 units) and sum
    uint32_t *seg_count;  // [B * H_kv * 2][kLineWords] pieces of a segment done so far; zero between launches
    int32_t n_wg, n_rseg, n_gseg;
    float scale, scale_log2e;
    uint16_t rmask[kMaxKvHeads];  // per KV head: bit i = query head g*group + i is a retrieval head
    uint8_t rhead[kMaxKvHeads];   // KV heads with a retrieval head,
    uint8_t ghead[kMaxKvHeads];   //   and with a sparse one
};

struct SelectArgs {
    PagedDims d;
    const float *scores;
    int64_t score_stride;
    const int32_t *lengths, *idx_in;
    int32_t *idx_out;
    uint64_t selects;  // bit g: KV head g's set is selected, else copied
};

// Partial slots of an attention launch, one a piece: pieces are at least an equal share of the blocks long, but for the
// last one of every segment ((request, KV head, kind of head)).
inline int64_t q4_slots(int32_t batch, int32_t n_segs, int32_t n_wg) { return (int64_t)batch * n_segs + n_wg; }

hipError_t launch_release(const ReleaseArgs &a, hipStream_t stream);
hipError_t launch_plan(const PlanArgs &a, hipStream_t stream);
hipError_t launch_append(const AppendArgs &a, hipStream_t stream);
hipError_t launch_read(const ReadArgs &a, hipStream_t stream);
hipError_t launch_q4_attn(const Q4AttnArgs &a, hipStream_t stream);
hipError_t launch_select(const SelectArgs &a, hipStream_t stream);

}  // namespace lychee
