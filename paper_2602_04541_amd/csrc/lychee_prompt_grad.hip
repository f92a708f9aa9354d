// Gradients of causal attention over packed sequences.
//
// With the notation of the forward pass (rows r are (query token, query head of the KV head), P_rj = 2^(s_rj - lse_r)) and g_r
// the gradient of out_r:
//     dP_rj = g_r . v_j,  delta_r = g_r . out_r,  dS_rj = P_rj (dP_rj - delta_r)
//     dq_r = c sum_j dS_rj k_j,  dk_j = c sum_r dS_rj q_r,  dv_j = sum_r P_rj g_r,  c = 1 / sqrt(128)
// Two launches, so that every sum is made in a fixed order and none needs atomics: the first goes over the keys of 128 rows, the second
// over the rows of 128 keys (all query heads of the KV head).  A wavefront makes a sum alone, or its range's part of one, and a merge
// adds the parts up, range after range.
// Scores and weights are made in both: seven products of a pair of tiles where five would do.
// P and dS are rounded to bf16 for the products that sum them, at most 2^-8 of each with either sign: as much again as the results' own
// rounding.  delta comes from the rounded out, which is all that the call has of it.
//
// What bounds it: the products and the registers.  8192 tokens of 32 heads (8 KV heads), forward and backward: 2.26 ms, of which
// the forward pass takes 0.52, dq 0.71 (three products: 1.17 PFLOP/s), dk and dv 1.01 (four: 1.09 PFLOP/s) and their merge 0.026.
// Sums of 128 keys and a block of scores fill the 256 registers of two wavefronts a unit, so K's rows stay in registers, V's in
// LDS, and 32 rows come at a time (64 at a time: 2.52 ms in all where 32 took 2.44).  No read of LDS meets a bank twice.
// Short: four launches, 49 us in all for four sequences of 93 to 311 tokens.
#include "lychee_prompt_device.h"

namespace lychee {
namespace {

// Reads of LDS ahead of their products: of the first products' rows, of the second's, and of V's rows where LDS has them.  (Eight
// thousand tokens: 2.26 ms forward and backward; 2.28 with four for the second, which leaves no registers to spare, 2.33 as the
// compiler places them.)
constexpr int kAhead = 4, kAheadTurned = 2, kAheadValues = 2;
constexpr int kPartFloats = 2 * 16 * 64 * 4;  // a wavefront's part of a range's sums
constexpr int kGradRows = 32;  // rows that the second launch takes at a time
constexpr int kGradBytes = kGradRows * kRowBytes;

struct SharedGrad {
    union {
        SharedPlan plan;  // (first launch, where a workgroup has a tile)
        struct {
            __align__(16) uint8_t a[2][kBlockBytes];
            __align__(16) uint8_t b[2][kBlockBytes];
            SharedLine line;
        };
        struct {
            __align__(16) uint8_t q[2][kGradBytes];
            __align__(16) uint8_t g[2][kGradBytes];
            __align__(16) float stat[2][2][kGradRows];  // of a block's rows: -lse sqrt(128), -delta
            __align__(16) bf16x8_t v[kWaves][8][64];
            SharedLine line;
        } keys;
    };
    int said[kWaves];  // (any_thread)
};
static_assert(sizeof(SharedGrad) <= 80 * 1024, "two workgroups a compute unit");

__device__ __forceinline__ float dot8(bf16x8_t a, bf16x8_t b, float acc)
{
    const u32x4_t x = __builtin_bit_cast(u32x4_t, a), y = __builtin_bit_cast(u32x4_t, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = dot2_bf16(x[i], y[i], acc);
    return acc;
}

// Sums of partials in their order, kBatch of them on their way at a time.
constexpr int kBatch = 8;
template <int N, typename At>
__device__ __forceinline__ void sum_parts(f32x4_t (&sum)[N], int parts, At at)
{
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int q = 0; q < parts; q += kBatch) {
        f32x4_t x[kBatch][N];
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                if (q + j < parts) x[j][i] = *(const LYCHEE_GLOBAL f32x4_t *)at(q + j, i);
            }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] += x[j][i];
    }
}

// dq, and lse and delta of every row for the second launch.  Scores and dP are made turned, as in the forward pass.
template <bool SHARE>
__global__ __launch_bounds__(kThreads, 2) void prompt_dq_kernel(PromptGradArgs a)
{
    __shared__ SharedGrad sh;
    const PromptRows &p = a.r;
    const int g = blockIdx.x % p.n_kv_heads;
    Work work;
    if (!begin_work<SHARE>(work, p, g, a.one_row_range, a.records, a.n_row_records, a.rows_by_number, sh.line, sh.plan)) return;
    if (!work.share) __syncthreads();  // (the plan's part of LDS is free)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    do {
        next_tile(work, p, g, a.records, a.n_row_records, a.rows_by_number, sh.line);
        const Tile w = work.w;
        const int lane = (int)opaque(threadIdx.x & 63), hi = lane >> 5;
        const int rows = w.n * p.group, first_row = w.tile * kPromptRows + wave * 32, row = first_row + (lane & 31);
        const int row_in = min(row, rows - 1), pos = token_of(p, row_in), head = g * p.group + row_in - pos * p.group;
        const int lowest = token_of(p, min(first_row, rows - 1));
        const int highest = first_row < rows ? token_of(p, min(first_row + 31, rows - 1)) : -1;  // (no rows: no products)
        const int64_t token = w.start + pos, packed = (token * (p.n_kv_heads * p.group) + head) * kHeadDim;
        const int64_t q_at = token * p.q_tok + (int64_t)head * p.q_head;

        bf16x8_t qf[8], gf[8];
        float delta = 0.f;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            qf[ks] = *(const LYCHEE_GLOBAL bf16x8_t *)(a.q + q_at + 16 * ks + 8 * hi);
            gf[ks] = *(const LYCHEE_GLOBAL bf16x8_t *)(a.g + packed + 16 * ks + 8 * hi);
            delta = dot8(gf[ks], *(const LYCHEE_GLOBAL bf16x8_t *)(a.out + packed + 16 * ks + 8 * hi), delta);
        }
        // What the products begin with, in units of q . k and of g . v
        const float less_delta = -sum_halves32(delta), less_lse = -gload(a.lse + (int64_t)head * p.n_tokens + token) * a.root;
        if (row < rows && hi == 0) {
            float *stat = a.stat + (int64_t)head * p.n_tokens + token;
            gstore(stat, less_lse);
            gstore(stat + (int64_t)p.n_kv_heads * p.group * p.n_tokens, less_delta);
        }

        const uint32_t row_at = row_place(lane), turn_at = turn_place(lane);
        const int64_t base = (int64_t)w.start * a.kv_tok + (int64_t)g * a.kv_head;
        const uint32_t to_k = lds_address(sh.a) + wave * 4 * kRowBytes, to_v = lds_address(sh.b) + wave * 4 * kRowBytes;
        const int fetch_row = 4 * wave + (lane >> 4);
        const uint32_t fetch_chunk = (uint32_t)((lane & 15) ^ swizzle(fetch_row)) << 4;
        const uint32_t fetch_at = (uint32_t)fetch_row * (uint32_t)(2 * a.kv_tok) + fetch_chunk;
        const auto fetch = [&](int blk, int buf) {
            const int j0 = blk * kPromptKeys;
            const bool whole = j0 + kPromptKeys <= w.len;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t from = base + (int64_t)(whole ? j0 + 16 * i : j0) * a.kv_tok;
                const uint32_t last = (uint32_t)min(fetch_row + 16 * i, w.len - 1 - j0);
                const uint32_t off = whole ? fetch_at : last * (uint32_t)(2 * a.kv_tok) + fetch_chunk;
                copy16(a.k + from, off, to_k + buf * kBlockBytes + i * 16 * kRowBytes);
                copy16(a.v + from, off, to_v + buf * kBlockBytes + i * 16 * kRowBytes);
            }
        };

        f32x16_t dq[4];
        bool careful = false;
        for (;;) {
            // with care, every block comes three times for either half of its keys (take_with_care)
            const int turns = (careful ? 6 : 1) * (w.last - w.first);
            const auto block_of = [&](int turn) { return w.first + (careful ? turn / 6 : turn); };
#pragma unroll
            for (int db = 0; db < 4; ++db) dq[db] = zero16();
            if (turns > 0) fetch(w.first, 0);
            arrived(qf);
            arrived(gf);
            wait_copies();
            __syncthreads();
            for (int turn = 0; turn < turns; ++turn) {
                const int blk = block_of(turn), buf = turn & 1, j0 = blk * kPromptKeys;
                if (turn + 1 < turns) fetch(block_of(turn + 1), buf ^ 1);
                const LYCHEE_LDS uint8_t *K = (const LYCHEE_LDS uint8_t *)sh.a[buf], *V = (const LYCHEE_LDS uint8_t *)sh.b[buf];
                if (careful || j0 <= highest) {
                    const bool masked = j0 + kPromptKeys - 1 > lowest;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (careful && turn % 2 != x) continue;
                        const uint32_t kat = opaque(row_at), vat = opaque(turn_at);
                        f32x16_t z = all16(less_lse), dp = all16(less_delta);
                        bf16x8_t first[kAhead], turned[kAheadTurned];  // read ahead of their products
                        uint32_t at = kat;
                        const auto read_first = [&](int i) {
                            if (i == 8) at = opaque(row_at);  // (addresses again, so that they need not be kept)
                            return read_rows(i < 8 ? K : V, at, x, i % 8);
                        };
                        const auto read_second = [&](int i) { return read_turned(K, vat, i % 4, 2 * x + i / 4); };
#pragma unroll
                        for (int i = 0; i < kAhead; ++i) first[i] = read_first(i);
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            in_order();
                            if (i < 8)
                                z = mfma(first[i % kAhead], qf[i], z);
                            else
                                dp = mfma(first[i % kAhead], gf[i - 8], dp);
                            if (i + kAhead < 16) first[i % kAhead] = read_first(i + kAhead);
                            if (i >= 16 - kAheadTurned) turned[i - (16 - kAheadTurned)] = read_second(i - (16 - kAheadTurned));
                            if (i >= 8) {  // (the weights while the other products go on)
                                z[2 * (i - 8)] = fast_exp2(z[2 * (i - 8)] * a.scale_log2e);
                                z[2 * (i - 8) + 1] = fast_exp2(z[2 * (i - 8) + 1] * a.scale_log2e);
                            }
                        }
                        in_order();
#pragma unroll
                        for (int i = 0; i < 16; ++i) z[i] *= dp[i];
                        if (masked) {
                            asm volatile("");
                            const int lim = pos - j0 - 32 * x - 4 * hi;
#pragma unroll
                            for (int i = 0; i < 16; ++i) z[i] = i % 4 + 8 * (i / 4) <= lim ? z[i] : 0.f;
                        }
                        bf16x8_t ds[2] = {operand<0>(z), operand<8>(z)};
                        if (__builtin_expect(careful, 0)) {
                            __syncthreads();
                            take_with_care(sh.a[buf], kBlockBytes, min(turn / 2 % 3, 1));
                            __syncthreads();
                            if (turn / 2 % 3 != 0) {
                                const uint32_t largest = turn / 2 % 3 == 1 ? kLargest : 0x8000u | kLargest;
#pragma unroll
                                for (int s = 0; s < 2; ++s) ds[s] = seen_rows(hi, 2 * x + s, 0, pos - j0, largest);
                            }
#pragma unroll
                            for (int i = 0; i < kAheadTurned; ++i) turned[i] = read_second(i);
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            in_order();
                            dq[i % 4] = mfma(turned[i % kAheadTurned], ds[i / 4], dq[i % 4]);
                            if (i + kAheadTurned < 8) turned[i % kAheadTurned] = read_second(i + kAheadTurned);
                        }
                        in_order();
                    }
                }
                wait_copies();
                __syncthreads();
            }
            if (careful || !any_thread(!all_finite(dq), wave, sh.said)) break;
            careful = true;
        }
        if (work.slot < 0) {
            store_row(row < rows ? a.dq + q_at : nullptr, lane, dq, a.scale);
        } else {
            store_part(a.part + (int64_t)(work.slot * kWaves + wave) * (kPartFloats / 2) + 4 * lane, dq);
        }
    } while (more_work(work));
}

// The sums of tiles that lie in several ranges, range after range: a workgroup has 32 rows, a wavefront every fourth group of
// eight dimensions, a lane four of a row.
__global__ __launch_bounds__(kThreads) void prompt_dq_merge_kernel(PromptGradArgs a)
{
    const PromptRows &p = a.r;
    const int g = blockIdx.x % p.n_kv_heads, unit = blockIdx.x / p.n_kv_heads, rows32 = unit % kWaves;
    const Record w = recorded(a.records, unit / kWaves);
    const int parts = w.parts, range = w.range;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rows = w.n * p.group;
    if (parts == 0 || w.tile * kPromptRows + rows32 * 32 >= rows) return;
    const int row = w.tile * kPromptRows + rows32 * 32 + (lane & 31), row_in = min(row, rows - 1);
    const int token = token_of(p, row_in), head = g * p.group + row_in - token * p.group;
    f32x4_t sum[4];
    sum_parts<4>(sum, parts, [&](int piece, int i) {
        const int64_t part = part_slot(range + piece, piece == 0, p.n_kv_heads, g) * kWaves + rows32;
        return a.part + part * (kPartFloats / 2) + (4 * i + wave) * 256 + 4 * lane;
    });
    if (row >= rows) return;
    uint16_t *to = a.dq + (int64_t)(w.start + token) * p.q_tok + (int64_t)head * p.q_head + 4 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < 4; ++i) store_four(to + 8 * (4 * i + wave), sum[i], a.scale);
}

// dk and dv.  A wavefront has 32 keys, whose rows of K stay in registers and of V in LDS, and goes over the rows that see them, 32 at a
// time: queries and output gradients in LDS, scores and dP with a lane for a key, so that P and dS are B operands of the sums over
// the rows.
__global__ __launch_bounds__(kThreads, 2) void prompt_dkv_kernel(PromptGradArgs a)
{
    __shared__ SharedGrad sh;
    const PromptRows &p = a.r;
    const int g = blockIdx.x % p.n_kv_heads;
    const Line line = lay_line<kLineKeys>(p, a.one_key_range, sh.keys.line);
    const int range = blockIdx.x / p.n_kv_heads;
    int64_t at = range * line.size;
    const int64_t until = min(at + line.size, line.all);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (g == 0) clear_records(a.records, a.n_key_records, a.keys_by_number, line, range);
    while (at < opaque64(until)) {
        const LineTile w = line_tile_at<kLineKeys>(p, at, line, sh.keys.line);
        const int64_t place = at - w.at, place_end = min(opaque64(until) - w.at, w.weight);
        if (place == 0 && g == 0) record_tile(a.records, a.n_key_records, a.keys_by_number, line, w, range, place_end == w.weight);
        at += place_end - place;
        const int tile = w.tile, rows = w.n * p.group;
        const int block = 2 * p.group * tile + (int)place, block_end = 2 * p.group * tile + (int)place_end;  // of its rows
        const int lane = (int)opaque(threadIdx.x & 63), hi = lane >> 5;
        const auto key_of = [&](uint32_t lane) { return tile * kPromptRows + wave * 32 + (int)(lane & 31); };
        const auto kv_of = [&](int key) { return (int64_t)(w.start + min(key, w.n - 1)) * a.kv_tok + (int64_t)g * a.kv_head; };
        const int64_t kv_at = kv_of(key_of(lane));
        bf16x8_t kf[8];
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            kf[ks] = *(const LYCHEE_GLOBAL bf16x8_t *)(a.k + kv_at + 16 * ks + 8 * hi);
            sh.keys.v[wave][ks][lane] = *(const LYCHEE_GLOBAL bf16x8_t *)(a.v + kv_at + 16 * ks + 8 * hi);
        }
        const uint32_t row_at = row_place(lane), turn_at = turn_place(lane);
        const uint32_t to_q = lds_address(sh.keys.q) + wave * 4 * kRowBytes, to_g = lds_address(sh.keys.g) + wave * 4 * kRowBytes;
        const int64_t packed_tok = (int64_t)p.n_kv_heads * p.group * kHeadDim;
        const auto fetch = [&](int r0, int buf) {
            const int t0 = token_of(p, r0), at = (int)opaque(lane);
            const int fetch_row = r0 + 4 * wave + (at >> 4);
            const uint32_t fetch_chunk = (uint32_t)((at & 15) ^ swizzle(fetch_row)) << 4;
            const uint16_t *q = a.q + (int64_t)(w.start + t0) * p.q_tok + (int64_t)g * p.group * p.q_head;
            const uint16_t *go = a.g + (int64_t)(w.start + t0) * packed_tok + (int64_t)g * p.group * kHeadDim;
#pragma unroll
            for (int i = 0; i < kGradRows / 16; ++i) {
                const int r = min(fetch_row + 16 * i, rows - 1), t = token_of(p, r), h = r - t * p.group;
                copy16(q, (uint32_t)(t - t0) * (uint32_t)(2 * p.q_tok) + (uint32_t)h * (uint32_t)(2 * p.q_head) + fetch_chunk,
                       to_q + buf * kGradBytes + i * 16 * kRowBytes);
                copy16(go, (uint32_t)(t - t0) * (uint32_t)(2 * packed_tok) + (uint32_t)h * (2 * kHeadDim) + fetch_chunk,
                       to_g + buf * kGradBytes + i * 16 * kRowBytes);
            }
            if (wave < 2 && at < kGradRows) {  // (one wavefront lse, one delta)
                const int r = min(r0 + at, rows - 1), t = token_of(p, r), h = r - t * p.group;
                copy4(a.stat + ((int64_t)wave * p.n_kv_heads + g) * p.group * p.n_tokens + w.start,
                      ((uint32_t)h * (uint32_t)p.n_tokens + (uint32_t)t) * 4u, lds_address(sh.keys.stat[buf][wave]));
            }
        };
        const auto arrive = [&]() {
            wait_copies();
            __syncthreads();
        };
        const int from = block * kPromptKeys, blocks = (min(block_end * kPromptKeys, rows) - from + kGradRows - 1) / kGradRows;
        const int wave_first = (tile * kPromptRows + wave * 32) * p.group;     // rows from here on see a key of the wavefront
        const int wave_all = (tile * kPromptRows + wave * 32 + 31) * p.group;  // and from here on all of them

        f32x16_t dk[4], dv[4];
        bool careful = false;
        for (;;) {
            const int turns = (careful ? 3 : 1) * blocks;  // (take_with_care)
            const auto row_of = [&](int turn) { return from + (careful ? turn / 3 : turn) * kGradRows; };
#pragma unroll
            for (int db = 0; db < 4; ++db) dk[db] = zero16(), dv[db] = zero16();
            fetch(row_of(0), 0);
            arrive();
            for (int turn = 0; turn < turns; ++turn) {
                const int r0 = row_of(turn), buf = turn & 1;
                if (turn + 1 < turns) fetch(row_of(turn + 1), buf ^ 1);
                const LYCHEE_LDS uint8_t *Q = (const LYCHEE_LDS uint8_t *)sh.keys.q[buf], *G = (const LYCHEE_LDS uint8_t *)sh.keys.g[buf];
                if (careful || r0 + kGradRows > wave_first) {
                    const uint32_t kat = opaque(row_at), vat = opaque(turn_at);
                    f32x16_t z, dp;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const f32x4_t l = *reinterpret_cast<const f32x4_t *>(&sh.keys.stat[buf][0][8 * j + 4 * hi]);
                        const f32x4_t d = *reinterpret_cast<const f32x4_t *>(&sh.keys.stat[buf][1][8 * j + 4 * hi]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) z[4 * j + i] = l[i], dp[4 * j + i] = d[i];
                    }
                    const auto least_of = [&]() { return key_of(opaque(lane)) * p.group - r0; };  // rows that see the lane's key
                    const int most = rows - 1 - r0;
                    // reads ahead of their products
                    bf16x8_t first[kAhead], vs[kAheadValues], turned[kAheadTurned];
                    uint32_t at = kat;
                    const auto read_first = [&](int i) {
                        if (i == 8) at = opaque(row_at);  // (addresses again, so that they need not be kept)
                        return read_rows(i < 8 ? Q : G, at, 0, i % 8);
                    };
                    const auto read_value = [&](int i) { return ((const LYCHEE_LDS bf16x8_t *)sh.keys.v[wave][i])[lane]; };
                    const auto read_second = [&](int i) { return read_turned(i < 8 ? G : Q, vat, i % 4, i / 4 % 2); };
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) first[i] = read_first(i);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        in_order();
                        z = mfma(first[i % kAhead], kf[i], z);
                        first[i % kAhead] = read_first(i + kAhead);
                        if (i >= 8 - kAheadValues) vs[i - (8 - kAheadValues)] = read_value(i - (8 - kAheadValues));
                    }
                    in_order();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {  // (the weights while these products go on)
                        in_order();
                        dp = mfma(first[(i + 8) % kAhead], vs[i % kAheadValues], dp);
                        if (i + kAhead < 8) first[(i + 8) % kAhead] = read_first(i + 8 + kAhead);
                        if (i + kAheadValues < 8) vs[i % kAheadValues] = read_value(i + kAheadValues);
                        if (i >= 8 - kAheadTurned) turned[i - (8 - kAheadTurned)] = read_second(i - (8 - kAheadTurned));
                        z[2 * i] = fast_exp2(z[2 * i] * a.scale_log2e);
                        z[2 * i + 1] = fast_exp2(z[2 * i + 1] * a.scale_log2e);
                        asm volatile("" : "+v"(z[2 * i]), "+v"(z[2 * i + 1]));
                    }
                    in_order();
#pragma unroll
                    for (int i = 0; i < 16; ++i) dp[i] *= z[i];
                    if (r0 < wave_all || r0 + kGradRows > rows) {
                        asm volatile("");
                        const int least = least_of();
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int r = i % 4 + 8 * (i / 4) + 4 * hi;
                            const bool seen = r >= least && r <= most;
                            z[i] = seen ? z[i] : 0.f;
                            dp[i] = seen ? dp[i] : 0.f;
                        }
                    }
                    bf16x8_t pf[2] = {operand<0>(z), operand<8>(z)}, ds[2] = {operand<0>(dp), operand<8>(dp)};
                    if (__builtin_expect(careful, 0)) {
                        __syncthreads();
                        take_with_care(sh.keys.q[buf], kGradBytes, turn % 3);
                        take_with_care(sh.keys.g[buf], kGradBytes, turn % 3);
                        __syncthreads();
                        if (turn % 3 != 0) {
#pragma unroll
                            for (int s = 0; s < 2; ++s) pf[s] = ds[s] = seen_rows(hi, s, least_of(), most);
                        }
#pragma unroll
                        for (int i = 0; i < kAheadTurned; ++i) turned[i] = read_second(i);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        in_order();
                        if (i < 8)
                            dv[i % 4] = mfma(turned[i % kAheadTurned], pf[i / 4], dv[i % 4]);
                        else
                            dk[i % 4] = mfma(turned[i % kAheadTurned], ds[i / 4 - 2], dk[i % 4]);
                        if (i + kAheadTurned < 16) turned[i % kAheadTurned] = read_second(i + kAheadTurned);
                    }
                    in_order();
                }
                arrive();
            }
            if (careful || !any_thread(!all_finite(dk) || !all_finite(dv), wave, sh.said)) break;
            careful = true;
        }
        if (place == 0 && place_end == w.weight) {
            const int key = key_of(opaque(lane));
            const int64_t to = kv_of(key);
            store_row(key < w.n ? a.dk + to : nullptr, lane, dk, a.scale);
            store_row(key < w.n ? a.dv + to : nullptr, lane, dv, 1.f);
        } else if (tile * kPromptRows + wave * 32 < w.n) {
            float *to = a.part + (part_slot(range, place == 0, p.n_kv_heads, g) * kWaves + wave) * kPartFloats + 4 * lane;
            store_part(to, dk);
            store_part(to + kPartFloats / 2, dv);
        }
    }
}

// The same for dk and dv: a workgroup has 32 keys of either.
__global__ __launch_bounds__(kThreads) void prompt_dkv_merge_kernel(PromptGradArgs a)
{
    const PromptRows &p = a.r;
    const int g = blockIdx.x % p.n_kv_heads, unit = blockIdx.x / p.n_kv_heads, of_v = unit % 2, keys32 = unit / 2 % kWaves;
    const Record w = recorded(a.records, unit / 2 / kWaves);
    const int parts = w.parts, range = w.range;
    if (parts == 0 || w.tile * kPromptRows + keys32 * 32 >= w.n) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, key = w.tile * kPromptRows + keys32 * 32 + (lane & 31);
    f32x4_t sum[4];
    sum_parts<4>(sum, parts, [&](int piece, int i) {
        const int64_t part = part_slot(range + piece, piece == 0, p.n_kv_heads, g) * kWaves + keys32;
        return a.part + part * kPartFloats + (16 * of_v + 4 * i + wave) * 256 + 4 * lane;
    });
    if (key >= w.n) return;
    uint16_t *to = (of_v ? a.dv : a.dk) + (int64_t)(w.start + key) * a.kv_tok + (int64_t)g * a.kv_head + 4 * (lane >> 5);
    const float f = of_v ? 1.f : a.scale;
#pragma unroll
    for (int i = 0; i < 4; ++i) store_four(to + 8 * (4 * i + wave), sum[i], f);
}

}  // namespace

hipError_t launch_prompt_grad(const PromptGradArgs &a, hipStream_t stream)
{
    const unsigned heads = (unsigned)a.r.n_kv_heads;
    if (a.n_row_ranges > 0) {
        const unsigned work = (unsigned)(a.n_row_ranges > a.n_row_tiles ? a.n_row_ranges : a.n_row_tiles);
        prompt_dq_kernel<true><<<work * heads, kThreads, 0, stream>>>(a);
        prompt_dq_merge_kernel<<<(unsigned)a.n_row_records * heads * kWaves, kThreads, 0, stream>>>(a);
    } else {
        prompt_dq_kernel<false><<<(unsigned)a.n_row_tiles * heads, kThreads, 0, stream>>>(a);
    }
    prompt_dkv_kernel<<<(unsigned)a.n_key_ranges * heads, kThreads, 0, stream>>>(a);
    if (a.n_key_ranges == 1) return hipGetLastError();  // (no tile lies in several)
    prompt_dkv_merge_kernel<<<(unsigned)a.n_key_records * heads * kWaves * 2, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace lychee
