// Gradients of causal attention over packed sequences.
//
// With the notation of the forward pass (rows r are (query token, query head of the KV head), P_rj = 2^(s_rj - lse_r)) and g_r
// the gradient of out_r:
//     dP_rj = g_r . v_j,  delta_r = g_r . out_r,  dS_rj = P_rj (dP_rj - delta_r)
//     dq_r = c sum_j dS_rj k_j,  dk_j = c sum_r dS_rj q_r,  dv_j = sum_r P_rj g_r,  c = 1 / sqrt(128)
// Two launches, so that every sum is made by one wavefront in a fixed order and none needs atomics: the first goes over the keys
// of 128 rows, the second over the rows of 128 keys (all query heads of the KV head, so that nothing is left to add up).
// Scores and weights are made in both: seven products of a pair of tiles where five would do.
#include "lychee_prompt_device.h"

namespace lychee {
namespace {

constexpr int kPartFloats = 2 * 16 * 64 * 4;  // a wavefront's part of a piece's sums
constexpr int kGradRows = 32;  // rows that the second launch takes at a time
constexpr int kGradBytes = kGradRows * kRowBytes;

struct SharedGrad {
    union {
        SharedPlan plan;
        struct {
            __align__(16) uint8_t a[2][kBlockBytes];
            __align__(16) uint8_t b[2][kBlockBytes];
        };
        struct {
            __align__(16) uint8_t q[2][kGradBytes];
            __align__(16) uint8_t g[2][kGradBytes];
            __align__(16) float stat[2][2][kGradRows];  // of a block's rows: -lse sqrt(128), -delta
            __align__(16) bf16x8_t v[kWaves][8][64];
            SharedLine line;
        } keys;
    };
};
static_assert(sizeof(SharedGrad) <= 80 * 1024, "two workgroups a compute unit");

__device__ __forceinline__ float dot8(bf16x8_t a, bf16x8_t b, float acc)
{
    const u32x4_t x = __builtin_bit_cast(u32x4_t, a), y = __builtin_bit_cast(u32x4_t, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = dot2_bf16(x[i], y[i], acc);
    return acc;
}

// dq, and lse and delta of every row for the second launch.  Scores and dP are made turned, as in the forward pass.
__global__ __launch_bounds__(kThreads, 2) void prompt_dq_kernel(PromptGradArgs a)
{
    __shared__ SharedGrad sh;
    const PromptRows &p = a.r;
    const int g = blockIdx.x % p.n_kv_heads;
    const Tile w = find_tile<false>(p, blockIdx.x / p.n_kv_heads, 0, sh.plan);
    if (!w.found) return;
    __syncthreads();  // (the plan's part of LDS is free)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hi = lane >> 5;
    const int rows = w.n * p.group, row = w.tile * kPromptRows + wave * 32 + (lane & 31);
    const int row_in = min(row, rows - 1), pos = token_of(p, row_in), head = g * p.group + row_in - pos * p.group;
    const int lowest = token_of(p, min(w.tile * kPromptRows + wave * 32, rows - 1));
    const int highest = token_of(p, min(w.tile * kPromptRows + wave * 32 + 31, rows - 1));
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
            const uint32_t off = whole ? fetch_at : (uint32_t)min(fetch_row + 16 * i, w.len - 1 - j0) * (uint32_t)(2 * a.kv_tok) + fetch_chunk;
            copy16(a.k + from, off, to_k + buf * kBlockBytes + i * 16 * kRowBytes);
            copy16(a.v + from, off, to_v + buf * kBlockBytes + i * 16 * kRowBytes);
        }
    };

    f32x16_t dq[4];
    bool careful = false;
    for (;;) {
        // with care, every block comes three times for either half of its keys (take_with_care)
        const int turns = careful ? 6 * w.last : w.last;
        const auto block_of = [&](int turn) { return careful ? turn / 6 : turn; };
#pragma unroll
        for (int db = 0; db < 4; ++db) dq[db] = zero16();
        fetch(0, 0);
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
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) {
                        z = mfma(read_rows(K, kat, x, ks), qf[ks], z);
                        dp = mfma(read_rows(V, kat, x, ks), gf[ks], dp);
                    }
                    __builtin_amdgcn_sched_group_barrier(kGroupRead, 6, 0);  // (reads ahead of their products)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        __builtin_amdgcn_sched_group_barrier(kGroupMfma, 1, 0);
                        if (i < 10) __builtin_amdgcn_sched_group_barrier(kGroupRead, 1, 0);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[i] = fast_exp2(z[i] * a.scale_log2e) * dp[i];
                    if (masked) {
                        const int lim = pos - j0 - 32 * x - 4 * hi;
#pragma unroll
                        for (int i = 0; i < 16; ++i) z[i] = i % 4 + 8 * (i / 4) <= lim ? z[i] : 0.f;
                    }
                    bf16x8_t ds[2] = {operand<0>(z), operand<8>(z)};
                    if (__builtin_expect(careful, 0)) {
                        __syncthreads();
                        take_with_care(sh.a[buf], kBlockBytes, turn / 2 % 3);
                        __syncthreads();
                        if (turn / 2 % 3 != 0) {
#pragma unroll
                            for (int s = 0; s < 2; ++s) ds[s] = seen_rows(hi, 2 * x + s, 0, pos - j0);
                        }
                    }
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int db = 0; db < 4; ++db) dq[db] = mfma(read_turned(K, vat, db, 2 * x + s), ds[s], dq[db]);
                    __builtin_amdgcn_sched_group_barrier(kGroupRead, 6, 0);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        __builtin_amdgcn_sched_group_barrier(kGroupMfma, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(kGroupRead, 2, 0);
                    }
                }
            }
            wait_copies();
            __syncthreads();
        }
        if (careful || !__syncthreads_or(!all_finite(dq))) break;
        careful = true;
    }
    store_row(row < rows ? a.dq + q_at : nullptr, lane, dq, a.scale);
}

// dk and dv.  A wavefront has 32 keys, whose rows of K and V stay in registers, and goes over the rows that see them, 64 at a time:
// queries and output gradients in LDS, scores and dP with a lane for a key, so that P and dS are B operands of the sums over
// the rows.
__global__ __launch_bounds__(kThreads, 2) void prompt_dkv_kernel(PromptGradArgs a)
{
    __shared__ SharedGrad sh;
    const PromptRows &p = a.r;
    const int g = blockIdx.x % p.n_kv_heads;
    const Line line = lay_line(p, a.n_ranges, sh.keys.line);
    const int range = blockIdx.x / p.n_kv_heads;
    int64_t at = range * line.size;
    const int64_t until = min(at + line.size, line.all);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    while (at < until) {
    const KeyTile w = tile_at(p, at, sh.keys.line);
    const int block = w.first + (int)(at - w.at), block_end = (int)min((int64_t)w.end, block + (until - at));
    const int tile = w.tile, rows = w.n * p.group;
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
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    z = mfma(read_rows(Q, kat, 0, ks), kf[ks], z);
                    dp = mfma(read_rows(G, kat, 0, ks), ((const LYCHEE_LDS bf16x8_t *)sh.keys.v[wave][ks])[lane], dp);
                }
                // (the first operands, and six reads ahead of the products from there)
                __builtin_amdgcn_sched_group_barrier(kGroupRead, 14, 0);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    __builtin_amdgcn_sched_group_barrier(kGroupMfma, 1, 0);
                    if (i % 2)
                        __builtin_amdgcn_sched_group_barrier(kGroupRead, 2, 0);
                    else
                        __builtin_amdgcn_sched_group_barrier(kGroupRead, 1, 0);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    z[i] = fast_exp2(z[i] * a.scale_log2e);
                    dp[i] *= z[i];
                }
                const auto least_of = [&]() { return key_of(opaque(lane)) * p.group - r0; };  // rows that see the lane's key
                const int most = rows - 1 - r0;
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
                }
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int db = 0; db < 4; ++db) {
                        dv[db] = mfma(read_turned(G, vat, db, s), pf[s], dv[db]);
                        dk[db] = mfma(read_turned(Q, vat, db, s), ds[s], dk[db]);
                    }
                __builtin_amdgcn_sched_group_barrier(kGroupRead, 8, 0);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    __builtin_amdgcn_sched_group_barrier(kGroupMfma, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kGroupRead, 2, 0);
                }
            }
            arrive();
        }
        if (careful || !__syncthreads_or(!all_finite(dk) || !all_finite(dv))) break;
        careful = true;
    }
    if (block == w.first && block_end == w.end) {
        const int key = key_of(opaque(lane));
        const int64_t to = kv_of(key);
        store_row(key < w.n ? a.dk + to : nullptr, lane, dk, a.scale);
        store_row(key < w.n ? a.dv + to : nullptr, lane, dv, 1.f);
    } else {
        // (of the two partials a range can leave the second is that of a tile's first blocks)
        const int64_t slot = ((int64_t)range * 2 + (block == w.first)) * p.n_kv_heads + g;
        float *to = a.part + (slot * kWaves + wave) * kPartFloats + 4 * lane;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                *(LYCHEE_GLOBAL f32x4_t *)(to + (4 * db + j) * 256) = f32x4_t{dk[db][4 * j], dk[db][4 * j + 1], dk[db][4 * j + 2], dk[db][4 * j + 3]};
                *(LYCHEE_GLOBAL f32x4_t *)(to + (16 + 4 * db + j) * 256) = f32x4_t{dv[db][4 * j], dv[db][4 * j + 1], dv[db][4 * j + 2], dv[db][4 * j + 3]};
            }
    }
    at += block_end - block;
    }
}

// The sums of tiles that lie in several ranges, range after range: a workgroup has 32 keys, a wavefront every fourth group of
// eight dimensions, a lane four of a key.
__global__ __launch_bounds__(kThreads) void prompt_dkv_merge_kernel(PromptGradArgs a)
{
    __shared__ SharedLine sh;
    __shared__ SharedPlan plan;
    const PromptRows &p = a.r;
    const int keys32 = blockIdx.x % kWaves, g = blockIdx.x / kWaves % p.n_kv_heads, number = blockIdx.x / kWaves / p.n_kv_heads;
    const Line line = lay_line(p, a.n_ranges, sh);
    int b = number < tiles_of(sh.n[0]) ? 0 : -1, tile = number;
    if (p.batch > 1) {
        const int t = threadIdx.x;
        find_request(p.batch, number, 0, t < p.batch ? tiles_of(sh.n[t]) : 0, 0, plan);
        b = plan.found[0];
        tile = plan.found[1];
    }
    b = __builtin_amdgcn_readfirstlane(b);
    if (b < 0) return;
    const KeyTile w = key_tile(p, b, __builtin_amdgcn_readfirstlane(tile), uniform64(sh.before[b]), sh);
    const int first = (int)(w.at / line.size), last = (int)((w.at + (w.end - w.first) - 1) / line.size);
    if (first == last || last >= a.n_ranges) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, key = w.tile * kPromptRows + keys32 * 32 + (lane & 31);
    const auto part_of = [&](int range, int second) {
        return a.part + ((((int64_t)range * 2 + second) * p.n_kv_heads + g) * kWaves + keys32) * kPartFloats + 4 * lane;
    };
    f32x4_t sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = *(const LYCHEE_GLOBAL f32x4_t *)(part_of(first, 1) + (4 * i + wave) * 256);
    for (int q = first + 1; q <= last; ++q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += *(const LYCHEE_GLOBAL f32x4_t *)(part_of(q, 0) + (4 * i + wave) * 256);
    }
    if (key >= w.n) return;
    const int64_t to = (int64_t)(w.start + key) * a.kv_tok + (int64_t)g * a.kv_head + 4 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int dj = (4 * i + wave) % 16;
        const float f = i < 4 ? a.scale : 1.f;
        *(LYCHEE_GLOBAL u32x2_t *)((i < 4 ? a.dk : a.dv) + to + 8 * dj) = u32x2_t{pk_bf16(sum[i][0] * f, sum[i][1] * f), pk_bf16(sum[i][2] * f, sum[i][3] * f)};
    }
}

}  // namespace

hipError_t launch_prompt_grad(const PromptGradArgs &a, hipStream_t stream)
{
    const unsigned heads = (unsigned)a.r.n_kv_heads;
    prompt_dq_kernel<<<(unsigned)a.n_row_tiles * heads, kThreads, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    prompt_dkv_kernel<<<(unsigned)a.n_ranges * heads, kThreads, 0, stream>>>(a);
    prompt_dkv_merge_kernel<<<(unsigned)a.n_key_tiles * heads * kWaves, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace lychee
