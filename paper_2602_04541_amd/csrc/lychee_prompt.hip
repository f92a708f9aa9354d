// Causal attention over whole prompts: packed rows of queries against keys that are packed alike, lie in a bf16 cache, or in
// the paged 4-bit cache.
//
// For row r of a (request, KV head) - query token t = r / G, query head r % G of the head's group - at position
// p = L - n + t:
//     s_j = q . k_j log2(e) / sqrt(128),  m = max s,  l = sum 2^(s_j - m),  o = sum 2^(s_j - m) v_j / l    over j <= p
// in one pass over blocks of 64 keys with a running m and l.
//
// A workgroup has 128 rows, 32 a wavefront, so that a KV head's keys are read once for all of its query heads and a single
// token's group shares a tile.  Scores are made turned, S^T = K Q^T: a lane has one row (column) and half of a
// block's keys, the running maximum and sum need one exchange between two lanes, and the weights are the B operand of the second
// product O^T = V^T P^T as they stand.
//
// What bounds it, long: the products, 64 of 32x32x16 for 128 rows and 64 keys, and the issue slots that are left between them.  16384
// tokens of 32 heads (8 KV heads) take 2.02 ms, 1.09 PFLOP/s; a library's product of 8192 x 8192 x 8192 reaches 1.30.  Power leaves
// either a clock of about 1.9 GHz, at which the matrix units could make 2.0: they are busy 55 to 57 % of the cycles here, 65 to 70 % in
// the library's product, which has no exponentials and sums to make.  No read of LDS meets a bank twice, and the same loop without its
// copies is 10 % faster.  Two wavefronts a unit share the rest: exponentials and sums of one beside the products of the other; the next
// block's scores begun beside a block's weights, weights made between products and priorities by wavefront all cost more than they
// gave.  Short: a launch and what it reads once, 6 us for 77 tokens.  Few rows over many keys: the memory's latency and the merge, 51 us
// for 32 rows over 32768 keys of 8 heads, of which the launch over the keys takes 43 (134 MB, 3.1 TB/s; 29 where the 256 MB
// last-level cache holds them) and the merge 8.5.
#include "lychee_prompt_device.h"

#include <type_traits>

namespace lychee {
namespace {

// Reads of keys ahead of their products (four, six and eight are as fast).  Of values eight are read before the weights are made, six of
// a 4-bit cache, whose next block is written into LDS between the last products: 6.69 ms for two pieces of 4001 to 4096 tokens that end
// at 32 K to 61 K (7.00 with the block written behind them).
constexpr int kAhead = 6;
constexpr float kSlack = 8.f;    // powers of two by which a score may exceed the maximum that weights are measured against
// The maximum of a row whose scores are all -infinity (sum 0, NaN), which is not taken for one that sees nothing (maximum -infinity; zero).
// Rows without a sum get it behind their last block: as the least maximum of every block it took 0.5 to 0.9 % of long calls.
constexpr float kLeast = -3.40282347e38f;
__device__ __forceinline__ float factor(float m, float l) { return l != 0.f ? 1.f / l : m == -__builtin_inff() ? 0.f : __builtin_nanf(""); }
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -__builtin_inff() : (m + __log2f(l)) * (1.f / kLog2e); }

struct SharedPrompt {
    __align__(16) uint8_t k[2][kBlockBytes];
    __align__(16) uint8_t v[2][kBlockBytes];
    __align__(8) uint16_t bad[2][kWaves];  // of a block's keys those whose page is not there, a bit each
    int said[kWaves];                      // (any_thread)
    union {
        SharedPlan plan;
        SharedLine line;
    };
};

// SHARE: a workgroup has a range of all tiles where lengths make it worth it (lay_line), else a tile like the other kernel's.
template <bool Q4, bool SHARE>
__global__ __launch_bounds__(kThreads, 2) void prompt_kernel(PromptArgs a)
{
    __shared__ SharedPrompt sh;
    constexpr int kAheadValues = Q4 ? 6 : 8;
    const PromptRows &p = a.r;
    const int g = blockIdx.x % p.n_kv_heads;
    Work work;
    if (!begin_work<SHARE>(work, p, g, a.one_range, a.records, a.n_records, a.by_number, sh.line, sh.plan)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    do {
        next_tile(work, p, g, a.records, a.n_records, a.by_number, sh.line);
        const Tile w = work.w;
        const int lane = (int)opaque(threadIdx.x & 63), hi = lane >> 5;
        const int rows = w.n * p.group, first_row = w.tile * kPromptRows + wave * 32, row = first_row + (lane & 31);
        const int row_in = min(row, rows - 1), token = token_of(p, row_in), head = g * p.group + row_in - token * p.group;
        const int pos = w.len - w.n + token;  // keys 0 .. pos are seen
        // Of the wavefront's rows.  One without rows makes no products: a token of 32 heads, 16 KV heads, over 25 K 4-bit keys takes
        // 41 us, 49 with them.
        const int lowest = w.len - w.n + token_of(p, min(first_row, rows - 1));
        const int highest = first_row < rows ? w.len - w.n + token_of(p, min(first_row + 31, rows - 1)) : -1;

        bf16x8_t qf[8];
        {
            const uint16_t *q = a.q + (int64_t)(w.start + token) * p.q_tok + (int64_t)head * p.q_head + 8 * hi;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) qf[ks] = *(const LYCHEE_GLOBAL bf16x8_t *)(q + 16 * ks);
        }
        const uint32_t row_at = row_place(lane), turn_at = turn_place(lane);

        // bf16: copies go to LDS as they are, 16 rows of either operand a step, four a wavefront.
        const int64_t base = p.lengths ? (int64_t)w.b * a.kv_batch : (int64_t)w.start * a.kv_tok;
        const uint16_t *kb = a.k + base + (int64_t)g * a.kv_head, *vb = a.v + base + (int64_t)g * a.kv_head;
        const uint32_t to_k = lds_address(sh.k) + wave * 4 * kRowBytes, to_v = lds_address(sh.v) + wave * 4 * kRowBytes;
        const int fetch_row = 4 * wave + (lane >> 4);
        const uint32_t fetch_chunk = (uint32_t)((lane & 15) ^ swizzle(fetch_row)) << 4;  // (the same for rows 16 apart)
        const uint32_t fetch_at = (uint32_t)fetch_row * (uint32_t)(2 * a.kv_tok) + fetch_chunk;
        uint32_t offset[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) offset[i] = fetch_at + (uint32_t)i * 32u * (uint32_t)a.kv_tok;
        const auto copy_rows = [&](const uint16_t *from, int blk, uint32_t to) {
            const uint16_t *at = from + (int64_t)(blk * kPromptKeys) * a.kv_tok;
            const int left = w.len - 1 - blk * kPromptKeys;
            if (left >= kPromptKeys - 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) copy16(at, offset[i], to + i * 16 * kRowBytes);
            } else {  // the last key again in the rows behind it
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    copy16(at, (uint32_t)min(fetch_row + 16 * i, left) * (uint32_t)(2 * a.kv_tok) + fetch_chunk, to + i * 16 * kRowBytes);
            }
        };
        // 4 bits: a wavefront takes a tile of 16 tokens of every block, a lane a quarter (one scale's dimensions) of a token's key and
        // of its value, whose bf16 numbers it writes.  (Writes go eight lanes at a time and meet a bank twice; in an order of tokens in
        // which none does they are no faster, 6.75 ms either way for the case above.)
        const int sub4 = lane & 15, part4 = lane >> 4;
        const uint32_t row4 = (uint32_t)(sub4 * kTokenBytes + 16 * part4), scale4 = (uint32_t)(kTileScales + part4 * kTileTokens + sub4);
        const uint32_t store_at = (uint32_t)((wave * 16 + sub4) * kRowBytes + (((4 * part4) ^ swizzle(sub4)) << 4));
        uint4 code_k = make_uint4(0, 0, 0, 0), code_v = code_k;
        uint32_t scale_k = 0, scale_v = 0;
        int entry = -1;  // of the block table, for the block that is loaded next
        const auto fetch_entry = [&](int blk) {
            const int token = min(blk * kPromptKeys + wave * kTileTokens, w.len - 1);
            return gload(a.table + (int64_t)w.b * a.d.table_stride + (token >> a.d.page_shift));
        };
        const auto load4 = [&](int blk) {  // (whether the tile's page is there)
            const int page = __builtin_amdgcn_readfirstlane(entry), tiles = 1 << (a.d.page_shift - 4);
            const bool there = (uint32_t)page < (uint32_t)a.d.n_pages;
            const int64_t number = (int64_t)(there ? page : 0) * a.d.page_tiles + (int64_t)g * tiles + ((blk * 4 + wave) & (tiles - 1));
            const uint8_t *tile = uniform(a.cache + number * kTileBytes);
            const u32x4_t k = *(const LYCHEE_GLOBAL u32x4_t *)((const LYCHEE_GLOBAL uint8_t *)tile + row4);
            const u32x4_t v = *(const LYCHEE_GLOBAL u32x4_t *)((const LYCHEE_GLOBAL uint8_t *)tile + 64 + row4);
            const uint32_t ks = *((const LYCHEE_GLOBAL uint8_t *)tile + scale4);
            const uint32_t vs = *((const LYCHEE_GLOBAL uint8_t *)tile + 4 * kTileTokens + scale4);
            code_k = make_uint4(k[0], k[1], k[2], k[3]);
            code_v = make_uint4(v[0], v[1], v[2], v[3]);
            const bool ok = there && blk * kPromptKeys + wave * kTileTokens + sub4 < w.len;
            scale_k = ok ? ks << 23 : 0u;  // (a scale of 0 makes numbers that are no NaN: a weight of 0 times NaN is NaN)
            scale_v = ok ? vs << 23 : 0u;
            return there;
        };
        const auto store4 = [&](uint8_t *block, uint4 code, uint32_t scale) {
            const float f = __builtin_bit_cast(float, scale);
            const uint32_t c4[4] = {code.x, code.y, code.z, code.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) *reinterpret_cast<uint4 *>(block + (store_at ^ (uint32_t)(c << 4))) = decode8(c4[c], f);
        };
        f32x16_t o[4];
        float m, l;
        constexpr int kNowhere = 0x7FFFFFFF;
        int there_from = kNowhere;  // Q4: the first key whose page is there
        bool careful = false;
        for (;;) {
            // Turns: a block each.  With care all blocks come three times (take_with_care): infinities are put back when all scores have
            // been seen and no sum is rescaled any more, by a factor that might round to zero.
            const int blocks = max(w.last - w.first, 0), turns = (careful ? 3 : 1) * blocks;
            const auto after = [&](int blk) { return blk + 1 == w.last ? w.first : blk + 1; };
            const auto fetch = [&](int blk, int turn) {
                if constexpr (Q4) {
                    const bool there = load4(blk);
                    if (lane == 0) sh.bad[turn & 1][wave] = there ? 0 : 0xFFFF;
                    entry = fetch_entry(after(blk));
                } else {
                    copy_rows(kb, blk, to_k + (turn & 1) * kBlockBytes);
                    copy_rows(vb, blk, to_v + (turn & 1) * kBlockBytes);
                }
            };
            const auto store_k = [&](int turn) { if constexpr (Q4) store4(sh.k[turn & 1], code_k, scale_k); };
            const auto store_v = [&](int turn) { if constexpr (Q4) store4(sh.v[turn & 1], code_v, scale_v); };
            const auto arrive = [&]() {
                if constexpr (!Q4) wait_copies();
                __syncthreads();
            };
#pragma unroll
            for (int db = 0; db < 4; ++db) o[db] = zero16();
            m = -__builtin_inff();
            l = 0.f;
            if (turns > 0) {
                if (Q4) entry = fetch_entry(w.first);
                fetch(w.first, 0);
            }
            arrived(qf);
            if (turns > 0) {
                store_k(0);
                store_v(0);
                arrive();
            }
            for (int turn = 0, blk = w.first; turn < turns; ++turn, blk = after(blk)) {
                const int j0 = blk * kPromptKeys;
                if (turn + 1 < turns) fetch(after(blk), turn + 1);
                if (careful || j0 <= highest) {
                    const LYCHEE_LDS uint8_t *K = (const LYCHEE_LDS uint8_t *)sh.k[turn & 1];
                    const LYCHEE_LDS uint8_t *V = (const LYCHEE_LDS uint8_t *)sh.v[turn & 1];
                    const uint32_t kat = opaque(row_at), vat = opaque(turn_at);
                    const bool again = careful && turn >= blocks;
                    if (__builtin_expect(careful, 0)) {
                        take_with_care(sh.v[turn & 1], kBlockBytes, turn / blocks);
                        __syncthreads();
                    }
                    f32x16_t z[2] = {zero16(), zero16()};
                    // read ahead of their products; the first values are on their way while the weights are made
                    bf16x8_t kf[kAhead], vf[kAheadValues];
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) kf[i] = read_rows(K, kat, i % 2, i / 2);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        in_order();
                        z[i % 2] = mfma(kf[i % kAhead], qf[i / 2], z[i % 2]);
                        if (i + kAhead < 16) kf[i % kAhead] = read_rows(K, kat, (i + kAhead) % 2, (i + kAhead) / 2);
                        const int early = i - (16 - kAheadValues);
                        if (early >= 0) vf[early] = read_turned(V, vat, early % 4, early / 4);
                    }
                    in_order();
                    uint64_t bad = 0;  // keys whose page is not there
                    if (Q4) {
                        const uint2 words = *reinterpret_cast<const uint2 *>(sh.bad[turn & 1]);
                        bad = (uint64_t)__builtin_amdgcn_readfirstlane(words.y) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane(words.x);
                        if (there_from == kNowhere && ~bad != 0) there_from = j0 + __builtin_ctzll(~bad);
                    }
                    if (j0 + kPromptKeys - 1 > lowest || bad != 0) {
                        asm volatile("");  // (a branch: these are many instructions, and rare)
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const int n = min(max(pos - j0 - 32 * x + 1, 0), 32);
                            uint32_t seen = n == 32 ? ~0u : (1u << n) - 1u;
                            if (Q4) seen &= ~(uint32_t)(bad >> (32 * x));
                            seen >>= 4 * hi;
#pragma unroll
                            for (int i = 0; i < 16; ++i) z[x][i] = seen >> (i % 4 + 8 * (i / 4)) & 1u ? z[x][i] : -__builtin_inff();
                        }
                    }
                    float top = z[0][0];
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 16; ++i) top = fmaxf(top, z[x][i]);
                    top = max_halves32(top) * a.scale_log2e;
                    // m is some maximum of late: weights of up to 2^kSlack are as exact as others, and a new maximum costs 65
                    // products.  (By the row's own scores alone, so that no row's bits depend on another's.)
                    if (__ballot(top > m + kSlack) != 0) {
                        asm volatile("");
                        const float up = top > m + kSlack ? top : m;
                        const float f = m == up ? 1.0f : fast_exp2(m - up);
                        m = up;
                        l *= f;
#pragma unroll
                        for (int db = 0; db < 4; ++db)
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[db][i] *= f;
                    }
                    const float ref = m == -__builtin_inff() ? 0.f : m;
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            z[x][i] = fast_exp2(__builtin_fmaf(z[x][i], a.scale_log2e, -ref));
                            part[i % 4] += z[x][i];
                        }
                    bf16x8_t pf[4] = {operand<0>(z[0]), operand<8>(z[0]), operand<0>(z[1]), operand<8>(z[1])};
                    if (__builtin_expect(again, 0)) {
#pragma unroll
                        for (int s = 0; s < 4; ++s) pf[s] = seen_rows(hi, s, 0, pos - j0);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        in_order();
                        o[i % 4] = mfma(vf[i % kAheadValues], pf[i / 4], o[i % 4]);
                        const int next = i + kAheadValues;
                        if (next < 16) vf[i % kAheadValues] = read_turned(V, vat, next % 4, next / 4);
                        if (i == 10) store_k(turn + 1);  // (the next block's numbers while the products go on)
                        if (i == 14) store_v(turn + 1);
                    }
                    l += again ? 0.f : (part[0] + part[1]) + (part[2] + part[3]);
                } else {
                    store_k(turn + 1);
                    store_v(turn + 1);
                }
                arrive();
            }
            // A key's value counts for the rows that see it alone, but a weight of zero times an infinite value or NaN is NaN: a
            // tile in which that may have happened is done again, with care.
            if (careful || !any_thread(!all_finite(o), wave, sh.said)) break;
            careful = true;
        }
        l = sum_halves32(l);
        if (l == 0.f && (Q4 ? there_from : w.first * kPromptKeys) <= min(pos, w.last * kPromptKeys - 1)) m = kLeast;  // (the row sees a key)
        if (work.slot < 0) {
            const bool there = row < rows;
            uint16_t *out = a.out + ((int64_t)(w.start + token) * (p.n_kv_heads * p.group) + head) * kHeadDim;
            store_row(there ? out : nullptr, lane, o, factor(m, l));
            if (a.lse && there && hi == 0) gstore(a.lse + (int64_t)head * p.n_tokens + w.start + token, lse_of(m, l));
        } else if (first_row < rows) {
            const int64_t part = (int64_t)work.slot * kWaves + wave;
            store_part(a.part_o + part * (64 * 64) + 4 * lane, o);
            if (hi == 0) gstore_f2(a.part_ml + (part * 32 + lane) * 2, make_float2(m, l));
        }
    } while (more_work(work));
}

// Rows of tiles that several ranges share: o = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p, M = max m_p.  A workgroup has 32 rows of
// a tile and some of the 16 groups of eight dimensions, its wavefronts a fourth of the pieces each, a lane four dimensions of a row, as
// the pieces left them; the wavefronts' sums meet in LDS.
// Pieces whose loads are in flight together; those of pieces that are not there are left out (all wavefronts at the last one's place
// instead: 10 us where 64 pieces of 8 heads take 8, and 54 where a call of 9 pieces takes 37).
constexpr int kMergeBatch = 16;
__global__ __launch_bounds__(kThreads) void prompt_merge_kernel(PromptArgs a)
{
    __shared__ __align__(16) f32x4_t sum[kWaves][64];
    __shared__ float2 ml[kWaves][64];
    const PromptRows &p = a.r;
    // (KV heads apart as in the launch before, whose partials lie in the caches of the same part of the device)
    const int g = blockIdx.x % p.n_kv_heads, unit = blockIdx.x / p.n_kv_heads;
    const int sub = unit % a.merge_split, rows32 = unit / a.merge_split % kWaves;
    const Record w = recorded(a.records, unit / a.merge_split / kWaves);
    const int parts = w.parts, range = w.range;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rows = w.n * p.group;
    if (parts == 0 || w.tile * kPromptRows + rows32 * 32 >= rows) return;
    const int row = w.tile * kPromptRows + rows32 * 32 + (lane & 31), row_in = min(row, rows - 1);
    const int token = token_of(p, row_in), head = g * p.group + row_in - token * p.group;
    const int64_t to = (int64_t)(w.start + token) * (p.n_kv_heads * p.group) + head;
    const auto at = [&](int piece) { return part_slot(range + piece, piece == 0, p.n_kv_heads, g) * kWaves + rows32; };
    const auto store = [&](int dj, f32x4_t o, float f) {  // (dimensions of register group dj: 32 db + 8 j + 4 hi)
        store_four(a.out + to * kHeadDim + 8 * dj + 4 * (lane >> 5), o, f);
    };
    const auto store_lse = [&](float m, float l) {
        if (a.lse && lane < 32) gstore(a.lse + (int64_t)head * p.n_tokens + w.start + token, lse_of(m, l));
    };
    // A piece's infinity stays one, though its weight may round to zero: sums that are no numbers are made again.
    const auto with_infinities = [&](f32x4_t o, int dj, float m) {
        const auto no_number = [](float x) { return !(__builtin_fabsf(x) < __builtin_inff()); };
        if (__builtin_expect(no_number(o[0]) || no_number(o[1]) || no_number(o[2]) || no_number(o[3]), 0)) {
            f32x4_t again = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int i = 0; i < parts; ++i) {
                const f32x4_t x = *(const LYCHEE_GLOBAL f32x4_t *)(a.part_o + at(i) * (64 * 64) + dj * 256 + 4 * lane);
                const float e = fast_exp2(gload(a.part_ml + (at(i) * 32 + (lane & 31)) * 2) - (m == -__builtin_inff() ? 0.f : m));
#pragma unroll
                for (int j = 0; j < 4; ++j) again[j] += (__builtin_isinf(x[j]) ? 1.f : e) * x[j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = no_number(o[j]) ? again[j] : o[j];
        }
        return o;
    };
    // Few pieces: a wavefront has all of them of a group of dimensions.
    const auto few = [&](auto most) {
        constexpr int kMost = decltype(most)::value;
        f32x2_t mls[kMost];
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            mls[i] = f32x2_t{-__builtin_inff(), 0.f};
            if (i < parts) mls[i] = *(const LYCHEE_GLOBAL f32x2_t *)(a.part_ml + (at(i) * 32 + (lane & 31)) * 2);
        }
        float m = -__builtin_inff(), l = 0.f, e[kMost];
#pragma unroll
        for (int i = 0; i < kMost; ++i) m = fmaxf(m, mls[i][0]);
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            e[i] = fast_exp2(mls[i][0] - (m == -__builtin_inff() ? 0.f : m));
            l += e[i] * mls[i][1];
        }
        if (sub == 0 && wave == 0 && row < rows) store_lse(m, l);
        for (int dj = sub * kWaves + wave; dj < 16; dj += a.merge_split * kWaves) {
            f32x4_t os[kMost], o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                os[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                if (i < parts) os[i] = *(const LYCHEE_GLOBAL f32x4_t *)(a.part_o + at(i) * (64 * 64) + dj * 256 + 4 * lane);
            }
#pragma unroll
            for (int i = 0; i < kMost; ++i) o += e[i] * os[i];
            if (row < rows) store(dj, with_infinities(o, dj, m), factor(m, l));
        }
    };
    if (parts <= 2) return few(std::integral_constant<int, 2>{});
    if (parts <= 4) return few(std::integral_constant<int, 4>{});
    if (parts <= 8) return few(std::integral_constant<int, 8>{});
    if (parts <= 16) return few(std::integral_constant<int, 16>{});
    for (int dj = sub; dj < 16; dj += a.merge_split) {
        float m = -__builtin_inff(), l = 0.f;
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
        for (int first = wave; first < parts; first += kWaves * kMergeBatch) {
            f32x2_t mls[kMergeBatch];
            f32x4_t os[kMergeBatch];
#pragma unroll
            for (int i = 0; i < kMergeBatch; ++i) {
                mls[i] = f32x2_t{-__builtin_inff(), 0.f};
                os[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                if (first + kWaves * i >= parts) continue;
                const int64_t from = at(first + kWaves * i);
                mls[i] = *(const LYCHEE_GLOBAL f32x2_t *)(a.part_ml + (from * 32 + (lane & 31)) * 2);
                os[i] = *(const LYCHEE_GLOBAL f32x4_t *)(a.part_o + from * (64 * 64) + dj * 256 + 4 * lane);
            }
            float up = m;
#pragma unroll
            for (int i = 0; i < kMergeBatch; ++i) up = fmaxf(up, mls[i][0]);
            const float ref = up == -__builtin_inff() ? 0.f : up, f = fast_exp2(m - ref);
            m = up;
            l *= f;
            o *= f;
#pragma unroll
            for (int i = 0; i < kMergeBatch; ++i) {
                const float e = fast_exp2(mls[i][0] - ref);
                l += e * mls[i][1];
                o += e * os[i];
            }
        }
        sum[wave][lane] = o;
        ml[wave][lane] = make_float2(m, l);
        __syncthreads();
        if (wave == 0) {
            float top = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < kWaves; ++i) top = fmaxf(top, ml[i][lane].x);
            const float ref = top == -__builtin_inff() ? 0.f : top;
            l = 0.f;
            o = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                const float e = fast_exp2(ml[i][lane].x - ref);
                l += e * ml[i][lane].y;
                o += e * sum[i][lane];
            }
            if (row < rows) {
                store(dj, with_infinities(o, dj, top), factor(top, l));
                if (dj == 0) store_lse(top, l);
            }
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_prompt(const PromptArgs &a, hipStream_t stream)
{
    const unsigned heads = (unsigned)a.r.n_kv_heads;
    if (a.n_ranges == 0) {
        if (a.cache)
            prompt_kernel<true, false><<<(unsigned)a.n_tiles * heads, kThreads, 0, stream>>>(a);
        else
            prompt_kernel<false, false><<<(unsigned)a.n_tiles * heads, kThreads, 0, stream>>>(a);
        return hipGetLastError();
    }
    const unsigned grid = (unsigned)(a.n_ranges > a.n_tiles ? a.n_ranges : a.n_tiles) * heads;
    if (a.cache)
        prompt_kernel<true, true><<<grid, kThreads, 0, stream>>>(a);
    else
        prompt_kernel<false, true><<<grid, kThreads, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    prompt_merge_kernel<<<(unsigned)a.n_records * heads * kWaves * (unsigned)a.merge_split, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace lychee
