// Device-side building blocks of attention over whole prompts: which tile a workgroup has, how rows and blocks of keys
// come to LDS, and how the matrix units take them from there.
//
// A matrix product here is v_mfma_f32_32x32x16_bf16, D[32][32] += A[32][16] B[16][32].  Lane (hi, n) = (lane / 32, lane % 32)
// holds A[n][8 hi ..+7], B[8 hi ..+7][n], and of D the column n: register i is row rows_of(i) = i%4 + 8 (i/4) + 4 hi.  A sum over
// 16 rows of one product's D therefore takes its B operand from D as it is, eight neighbouring registers a lane: the lane
// then has rows 16 s + 4 hi + {0..3} and 16 s + 8 + 4 hi + {0..3}, and the A operand is read in the same order.
//
// In LDS a block is 64 rows of 256 bytes, 16 chunks of 16 bytes, chunk c of row r at place c ^ swizzle(r).  LDS serves 256 bytes
// a cycle: along the rows (ds_read_b128, lane n its row's chunk) 16 rows, which are in 16 places; across them
// (ds_read_b64_tr_b16, 16 lanes take 4 rows of two neighbouring chunks and turn them) four rows of four chunks, in 16 places
// too.  Neither meets a bank twice.
#pragma once
#include "lychee_device.h"
#include "lychee_prompt.h"

namespace lychee {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
#define LYCHEE_LDS __attribute__((address_space(3)))

constexpr int kGroupMfma = 0x8, kGroupRead = 0x100;  // kinds of instructions, for the scheduler: matrix products, reads of LDS
constexpr int kRowBytes = 2 * kHeadDim;
constexpr int kBlockBytes = kPromptKeys * kRowBytes;

__device__ __forceinline__ int swizzle(int row) { return (row & 3) << 2 | ((row >> 2) & 3); }

__device__ __forceinline__ f32x16_t mfma(bf16x8_t a, bf16x8_t b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ uint32_t pk_bf16(float a, float b)  // round to nearest even, a in the low half
{
    bf16x2_t r;
    r[0] = (__bf16)a;
    r[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, r);
}

// Eight codes of the 4-bit cache as bf16 numbers, exactly; scale: a float with the scale byte as its exponent.
__device__ __forceinline__ uint4 decode8(uint32_t c, float scale)
{
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3)));
}

// Eight neighbouring registers of a product's D as the B operand of the next.  The rounding to bf16 is one of 2^-9 of a
// number at most, with either sign, like that of the output.
template <int kFirst>
__device__ __forceinline__ bf16x8_t operand(const f32x16_t &d)
{
    return __builtin_bit_cast(bf16x8_t, u32x4_t{pk_bf16(d[kFirst], d[kFirst + 1]), pk_bf16(d[kFirst + 2], d[kFirst + 3]),
                                               pk_bf16(d[kFirst + 4], d[kFirst + 5]), pk_bf16(d[kFirst + 6], d[kFirst + 7])});
}

__device__ __forceinline__ f32x16_t all16(float x)
{
    f32x16_t z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = x;
    return z;
}
__device__ __forceinline__ f32x16_t zero16() { return all16(0.f); }

// ------------------------------------------------------------------------------ rows
__device__ __forceinline__ int token_of(const PromptRows &p, int row) { return p.group == 1 ? row : (int)__umulhi((uint32_t)row, p.group_magic); }

// What a workgroup works on: a piece of a tile, which is kPromptRows rows of a (request, KV head).
struct Tile {
    int b, tile;
    int n, len;            // query tokens and keys of the request
    int start;             // its first token among the packed rows
    int piece, parts;      // this piece and how many the tile has that hold keys (at least 1)
    int first, last;       // blocks of keys of the piece
    int slot;              // of the piece's partial in its KV head (in a merge: of the tile's first piece)
    bool found;
};

struct SharedPlan {
    int32_t n[kMaxBatch], len[kMaxBatch], start[kMaxBatch], weight[kMaxBatch];
    int32_t items[kMaxBatch], slots[kMaxBatch];  // by rank
    uint8_t who[kMaxBatch];                      // the request of a rank
    uint32_t wave[2][kWaves];
    unsigned long long work[kWaves];
    int32_t found[3];
};
static_assert(kThreads == kMaxBatch, "a thread a request");

__device__ __forceinline__ void request_of(const PromptRows &p, int b, int &start, int &n, int &len)
{
    const int from = min(max(gload(p.start + b), 0), p.n_tokens), to = min(gload(p.start + b + 1), p.n_tokens);
    start = from;
    n = max(to - from, 0);
    len = p.lengths ? min(max(gload(p.lengths + b), 0), p.max_len) : n;
}
__device__ __forceinline__ int blocks_of(int keys) { return (int)(((int64_t)keys + kPromptKeys - 1) / kPromptKeys); }
__device__ __forceinline__ int tiles_of(int rows) { return (rows + kPromptRows - 1) / kPromptRows; }

// Sum over the workgroup's threads, for all of them.
__device__ __forceinline__ unsigned long long sum_all(unsigned long long w, SharedPlan &sh)
{
    for (int d = 32; d > 0; d >>= 1) w += __shfl_xor(w, d);
    if ((threadIdx.x & 63) == 0) sh.work[threadIdx.x >> 6] = w;
    __syncthreads();
    w = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) w += sh.work[i];
    return w;
}

// Which request has the `number`th of all the requests' `items`, where thread b knows request b's numbers of items and of `slots`
// for partials.  Requests come in descending order of `weight`, so that what takes longest begins first.  The answer
// is sh.found: the request or -1, the number within it, the slots of the requests before it.
__device__ __forceinline__ void find_request(int batch, int number, int weight, int items, int slots, SharedPlan &sh)
{
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    sh.weight[t] = weight;
    if (t == 0) sh.found[0] = -1;
    __syncthreads();
    int rank = t;
    if (batch > 1) {
        rank = 0;
        for (int i = 0; i < batch; ++i) {
            const int other = sh.weight[i];
            rank += other > weight || (other == weight && i < t);
        }
    }
    if (t < batch) {
        sh.items[rank] = items;
        sh.slots[rank] = slots;
        sh.who[rank] = (uint8_t)t;
    }
    __syncthreads();
    const uint32_t items_here = t < batch ? (uint32_t)sh.items[t] : 0u, slots_here = t < batch ? (uint32_t)sh.slots[t] : 0u;
    const uint32_t items_upto = wave_scan(items_here), slots_upto = wave_scan(slots_here);
    if (lane == 63) {
        sh.wave[0][wave] = items_upto;
        sh.wave[1][wave] = slots_upto;
    }
    __syncthreads();
    uint32_t items_before = items_upto - items_here, slots_before = slots_upto - slots_here;
    for (int i = 0; i < wave; ++i) {
        items_before += sh.wave[0][i];
        slots_before += sh.wave[1][i];
    }
    if ((uint32_t)number - items_before < items_here) {
        sh.found[0] = sh.who[t];
        sh.found[1] = number - (int)items_before;
        sh.found[2] = (int)slots_before;
    }
    __syncthreads();
}

// A request that a workgroup has found a piece of: the piece's number within it, and its first partial's.
struct Found {
    int b, at, before, start, n, len;
};
__device__ __forceinline__ Found found_alone(int number, int items, int start, int n, int len)
{
    Found f;
    f.b = number < __builtin_amdgcn_readfirstlane(items) ? 0 : -1;
    f.at = number;
    f.before = 0;
    f.start = __builtin_amdgcn_readfirstlane(start);
    f.n = __builtin_amdgcn_readfirstlane(n);
    f.len = __builtin_amdgcn_readfirstlane(len);
    return f;
}
__device__ __forceinline__ Found found_among(const SharedPlan &sh)
{
    Found f;
    f.b = __builtin_amdgcn_readfirstlane(sh.found[0]);
    f.at = __builtin_amdgcn_readfirstlane(sh.found[1]);
    f.before = __builtin_amdgcn_readfirstlane(sh.found[2]);
    const int b = f.b < 0 ? 0 : f.b;
    f.start = __builtin_amdgcn_readfirstlane(sh.start[b]);
    f.n = __builtin_amdgcn_readfirstlane(sh.n[b]);
    f.len = __builtin_amdgcn_readfirstlane(sh.len[b]);
    return f;
}

// The piece with this number (MERGE: the tile); of a request the last tile first, which sees most keys.  `slots` > 0: tiles are
// split into pieces of so many blocks that there are about `slots` of them in all KV heads.
template <bool MERGE>
__device__ __forceinline__ Tile find_tile(const PromptRows &p, int number, int slots, SharedPlan &sh)
{
    const bool alone = p.batch == 1;  // (nothing to look for, no barrier)
    const int t = alone ? 0 : threadIdx.x;
    int start = 0, n = 0, len = 0;
    if (t < p.batch) request_of(p, t, start, n, len);
    const int tiles = tiles_of(n * p.group), blocks = blocks_of(len);
    int size = 1 << 30;
    if (slots > 0) {
        unsigned long long w = (unsigned long long)tiles * (unsigned)max(blocks, 1) * (unsigned)p.n_kv_heads;
        if (!alone) w = sum_all(w, sh);
        size = __builtin_amdgcn_readfirstlane(max((int)min((w + slots - 1) / slots, 1ull << 30), kPromptMinPiece));
    }
    const int items = tiles * max(1, (blocks + size - 1) / size);
    Found f;
    if (alone) {
        f = found_alone(number, MERGE ? tiles : items, start, n, len);
    } else {
        sh.n[t] = n;
        sh.len[t] = len;
        sh.start[t] = start;
        find_request(p.batch, number, len, MERGE ? tiles : items, items, sh);
        f = found_among(sh);
    }
    Tile w;
    w.b = f.b;
    w.found = f.b >= 0;
    if (!w.found) return w;
    w.n = f.n;
    w.len = f.len;
    w.start = f.start;
    const int rows = w.n * p.group, pieces = max(1, (blocks_of(w.len) + size - 1) / size);
    w.tile = tiles_of(rows) - 1 - (MERGE ? f.at : f.at / pieces);
    w.piece = MERGE ? 0 : f.at % pieces;
    w.slot = f.before + (MERGE ? f.at * pieces : f.at);
    const int seen = max(0, w.len - w.n + token_of(p, min((w.tile + 1) * kPromptRows, rows) - 1) + 1);  // keys of the last row
    w.parts = max(1, (blocks_of(seen) + size - 1) / size);
    w.first = pieces == 1 ? 0 : w.piece * size;
    w.last = min(blocks_of(seen), pieces == 1 ? 1 << 30 : w.first + size);
    return w;
}

// Tiles of kPromptRows keys, which the rows from the tile's first key on see, as a line of blocks of kPromptKeys rows:
// request after request and tile after tile.  Tile k of a request with `end` blocks of rows has end - 2 G k of them.  A
// workgroup has a range of the line, all of the same size, whatever tiles it holds the parts of.
__device__ __forceinline__ int64_t blocks_before(int64_t tile, int end, int group) { return tile * end - (int64_t)group * tile * (tile - 1); }

struct SharedLine {
    int32_t n[kMaxBatch], start[kMaxBatch];
    int64_t before[kMaxBatch];  // blocks of the requests before
    int64_t wave[kWaves];
};
struct Line {
    int64_t all, size;  // blocks of the line, and of a range
};
__device__ __forceinline__ int64_t uniform64(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}
__device__ __forceinline__ Line lay_line(const PromptRows &p, int ranges, SharedLine &sh)
{
    static_assert(kPromptRows == 2 * kPromptKeys, "");
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    int start = 0, n = 0, len = 0;
    if (t < p.batch) request_of(p, t, start, n, len);
    const int64_t work = blocks_before(tiles_of(n), blocks_of(n * p.group), p.group);
    int64_t upto = work;
    if (p.batch > 1) {
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t x = __shfl_up(upto, d);
            upto += lane >= d ? x : 0;
        }
        if (lane == 63) sh.wave[wave] = upto;
        __syncthreads();
        for (int i = 0; i < wave; ++i) upto += sh.wave[i];
    }
    sh.n[t] = n;
    sh.start[t] = start;
    sh.before[t] = upto - work;
    __syncthreads();
    Line l;
    const int last = p.batch - 1, n_last = sh.n[last];
    l.all = uniform64(sh.before[last] + blocks_before(tiles_of(n_last), blocks_of(n_last * p.group), p.group));
    l.size = max((l.all + ranges - 1) / ranges, (int64_t)kPromptMinRowPiece);
    return l;
}

struct KeyTile {
    int n, start, tile;
    int64_t at;       // of its first block on the line
    int first, end;   // its blocks of rows
};
__device__ __forceinline__ KeyTile key_tile(const PromptRows &p, int b, int tile, int64_t before, const SharedLine &sh)
{
    KeyTile k;
    k.n = __builtin_amdgcn_readfirstlane(sh.n[b]);
    k.start = __builtin_amdgcn_readfirstlane(sh.start[b]);
    k.end = blocks_of(k.n * p.group);
    k.tile = tile;
    k.first = 2 * p.group * tile;
    k.at = before + blocks_before(tile, k.end, p.group);
    return k;
}
// The tile that holds a block of the line.
__device__ __forceinline__ KeyTile tile_at(const PromptRows &p, int64_t at, const SharedLine &sh)
{
    int b = 0;
    for (int step = kMaxBatch / 2; step > 0; step >>= 1)
        if (b + step < p.batch && uniform64(sh.before[b + step]) <= at) b += step;
    const int64_t before = uniform64(sh.before[b]);
    const int n = __builtin_amdgcn_readfirstlane(sh.n[b]), end = blocks_of(n * p.group), tiles = tiles_of(n);
    int tile = 0;
    for (int step = tiles > 1 ? 1 << (31 - __builtin_clz(tiles - 1)) : 0; step > 0; step >>= 1)
        if (tile + step < tiles && blocks_before(tile + step, end, p.group) <= at - before) tile += step;
    return key_tile(p, b, tile, before, sh);
}

// ------------------------------------------------------------------------------ LDS
// Sixteen bytes a lane from global memory to LDS, lane after lane from `to` on (base and to: the same for the wavefront).  In
// assembly, because the compiler lets every later read of LDS wait for such a copy at once, whichever part of LDS it writes; the
// kernels wait themselves, before the barrier behind which the copied block is read.
template <typename T>
__device__ __forceinline__ const T *uniform(const T *p)  // (in scalar registers, whatever the compiler knows of it)
{
    const uint64_t u = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const T *>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)u));
}
__device__ __forceinline__ void copy16(const uint16_t *base, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane((int)to)), "v"(offset), "s"(uniform(base)) : "memory");
}
__device__ __forceinline__ void copy4(const float *base, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(__builtin_amdgcn_readfirstlane((int)to)), "v"(offset), "s"(uniform(base)) : "memory");
}
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(const LYCHEE_LDS uint8_t *)p; }

// The A operand of step `ks` (16 dimensions) of a block's rows 32 x ..+31: lane's place for step 0 (row_place), which
// steps change in the chunk's bits alone.
__device__ __forceinline__ uint32_t row_place(int lane)
{
    const int row = lane & 31;
    return (uint32_t)(row * kRowBytes + (((lane >> 5) ^ swizzle(row)) << 4));
}
__device__ __forceinline__ bf16x8_t read_rows(const LYCHEE_LDS uint8_t *block, uint32_t place, int x, int ks)
{
    return *(const LYCHEE_LDS bf16x8_t *)(block + x * 32 * kRowBytes + (place ^ (uint32_t)(ks << 5)));
}

// The A operand of a block turned: rows are dimensions 32 db ..+31, columns the block's rows 16 s + 4 hi + {0..3} and
// 16 s + 8 + 4 hi + {0..3}.
__device__ __forceinline__ uint32_t turn_place(int lane)
{
    const int j = lane & 15, row = 4 * (lane >> 5) + (j >> 2), chunk = 2 * ((lane >> 4) & 1) + ((j >> 1) & 1);
    return (uint32_t)(row * kRowBytes + ((chunk ^ swizzle(row)) << 4) + (j & 1) * 8);
}
__device__ __forceinline__ bf16x8_t read_turned(const LYCHEE_LDS uint8_t *block, uint32_t place, int db, int s)
{
    const LYCHEE_LDS uint8_t *p = block + s * 16 * kRowBytes;
    const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LYCHEE_LDS s16x4_t *)(p + (place ^ (uint32_t)(db << 6))));
    const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LYCHEE_LDS s16x4_t *)(p + 8 * kRowBytes + (place ^ (uint32_t)(db << 6 | 32))));
    typedef short s16x8_t __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8_t, (s16x8_t)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
// A number the compiler forgets what it is made of: what derives from it is computed where it is used, an instruction each, and
// kept in no register from block to block.
__device__ __forceinline__ uint32_t opaque(uint32_t x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// Pairs that must not count have a weight of zero, but zero times an infinity or NaN is NaN.  A workgroup whose sums hold
// no numbers makes them again with care, every block three times: with zeros for such values (turn 0), and then with finite numbers
// that put them back where they count.  The largest bf16 number, squared, is an infinity in fp32: turn 1 has it, with its
// sign, for infinities and NaN, the products' other operand being that number for the pairs that count and zero for the others
// (seen_rows), and turn 2 its negative for NaN, which both infinities add up to.  The block is changed in LDS, behind the products
// that make the scores.
constexpr uint32_t kLargest = 0x7F7Fu;
__device__ __forceinline__ void take_with_care(uint8_t *block, int bytes, int turn)
{
#pragma unroll 1
    for (int i = threadIdx.x; i < bytes / 4; i += kThreads) {
        uint32_t *at = reinterpret_cast<uint32_t *>(block) + i, both = *at, to = 0;
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
            const uint32_t x = both >> h & 0xFFFFu, size = x & 0x7FFFu;
            uint32_t y = size < 0x7F80u ? x : 0u;
            if (turn == 1) y = size < 0x7F80u ? 0u : size > 0x7F80u ? kLargest : (x & 0x8000u) | kLargest;
            if (turn == 2) y = size > 0x7F80u ? 0x8000u | kLargest : 0u;
            to |= y << h;
        }
        *at = to;
    }
}
// The pairs that count, of step s in the order of read_turned: rows least .. most of the block's.
__device__ __forceinline__ bf16x8_t seen_rows(int hi, int s, int least, int most)
{
    u32x4_t u;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int row = 16 * s + 4 * hi + (w & 1) * 2 + (w >> 1) * 8;
        u[w] = (row >= least && row <= most ? kLargest : 0u) | (row + 1 >= least && row + 1 <= most ? kLargest << 16 : 0u);
    }
    return __builtin_bit_cast(bf16x8_t, u);
}

__device__ __forceinline__ bool all_finite(const f32x16_t (&x)[4])
{
    float bad = 0.f;  // (a number times zero is zero unless it is infinite or NaN)
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) bad = __builtin_fmaf(x[d][i], 0.f, bad);
    return bad == 0.f;
}

// A product's D, transposed rows of 128 numbers: column n is row n, registers of db its dimensions 32 db ..+31.  Sixteen bytes a
// lane: two lanes exchange halves, so that each has eight neighbouring dimensions.
__device__ __forceinline__ void store_row(uint16_t *row, int lane, const f32x16_t (&x)[4], float f)
{
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            u32x4_t u;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int i = 8 * j + 2 * w;
                const auto r = __builtin_amdgcn_permlane32_swap(pk_bf16(x[db][i] * f, x[db][i + 1] * f),
                                                                pk_bf16(x[db][i + 4] * f, x[db][i + 5] * f), false, false);
                u[w] = (uint32_t)r[0];
                u[2 + w] = (uint32_t)r[1];
            }
            if (row) *(LYCHEE_GLOBAL u32x4_t *)(row + 32 * db + 16 * j + 8 * (lane >> 5)) = u;
        }
}

}  // namespace
}  // namespace lychee
