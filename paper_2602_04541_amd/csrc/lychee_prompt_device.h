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

constexpr int kRowBytes = 2 * kHeadDim;
constexpr int kBlockBytes = kPromptKeys * kRowBytes;

__device__ __forceinline__ int swizzle(int row) { return (row & 3) << 2 | ((row >> 2) & 3); }

__device__ __forceinline__ f32x16_t mfma(bf16x8_t a, bf16x8_t b, f32x16_t c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

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

// Eight neighbouring registers of a product's D as the B operand of the next.  The rounding to bf16 is one of 2^-8 of a
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
__device__ __forceinline__ int token_of(const PromptRows &p, int row)
{
    return p.group == 1 ? row : (int)__umulhi((uint32_t)row, p.group_magic);
}

// What a workgroup works on: blocks of keys of a tile, which is kPromptRows rows of a (request, KV head).
struct Tile {
    int b, tile;
    int n, len;       // query tokens and keys of the request
    int start;        // its first token among the packed rows
    int first, last;  // blocks of keys
    bool found;
};

struct SharedPlan {
    int32_t n[kMaxBatch], len[kMaxBatch], start[kMaxBatch], weight[kMaxBatch];
    int32_t tiles[kMaxBatch];  // by rank
    uint8_t who[kMaxBatch];    // the request of a rank
    uint32_t wave[kWaves];
    int32_t found[2];
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
__device__ __forceinline__ int blocks_seen(const PromptRows &p, int tile, int n, int len)  // by a tile's last row
{
    return blocks_of(max(0, len - n + token_of(p, min((tile + 1) * kPromptRows, n * p.group) - 1) + 1));
}

__device__ __forceinline__ int64_t uniform64(int64_t x)
{
    const uint32_t high = (uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32));
    return (int64_t)((uint64_t)high << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// Which request has the `number`th of all the requests' tiles, where thread b knows request b's `tiles`.  Requests come in
// descending order of `weight`, so that what takes longest begins first.  The answer is sh.found: the request or -1, and the
// number within it.
__device__ __forceinline__ void find_request(int batch, int number, int weight, int tiles, SharedPlan &sh)
{
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    sh.weight[t] = weight;
    if (t == 0) sh.found[0] = -1;
    __syncthreads();
    int rank = 0;
    for (int i = 0; i < batch; ++i) {
        const int other = sh.weight[i];
        rank += other > weight || (other == weight && i < t);
    }
    if (t < batch) {
        sh.tiles[rank] = tiles;
        sh.who[rank] = (uint8_t)t;
    }
    __syncthreads();
    const uint32_t here = t < batch ? (uint32_t)sh.tiles[t] : 0u, upto = wave_scan(here);
    if (lane == 63) sh.wave[wave] = upto;
    __syncthreads();
    uint32_t before = upto - here;
    for (int i = 0; i < wave; ++i) before += sh.wave[i];
    if ((uint32_t)number - before < here) {
        sh.found[0] = sh.who[t];
        sh.found[1] = number - (int)before;
    }
    __syncthreads();
}

// The tile with this number, all its blocks; of a request the last tile first, which sees most keys.
__device__ __forceinline__ Tile find_tile(const PromptRows &p, int number, SharedPlan &sh)
{
    const bool alone = p.batch == 1;  // (nothing to look for, no barrier)
    const int t = alone ? 0 : threadIdx.x;
    int start = 0, n = 0, len = 0;
    if (t < p.batch) request_of(p, t, start, n, len);
    const int tiles = tiles_of(n * p.group);
    Tile w;
    int at = number;
    if (alone) {
        w.b = number < __builtin_amdgcn_readfirstlane(tiles) ? 0 : -1;
    } else {
        sh.n[t] = n;
        sh.len[t] = len;
        sh.start[t] = start;
        find_request(p.batch, number, len, tiles, sh);
        w.b = __builtin_amdgcn_readfirstlane(sh.found[0]);
        at = __builtin_amdgcn_readfirstlane(sh.found[1]);
        const int b = w.b < 0 ? 0 : w.b;
        start = sh.start[b];
        n = sh.n[b];
        len = sh.len[b];
    }
    w.found = w.b >= 0;
    if (!w.found) return w;
    w.start = __builtin_amdgcn_readfirstlane(start);
    w.n = __builtin_amdgcn_readfirstlane(n);
    w.len = __builtin_amdgcn_readfirstlane(len);
    w.tile = tiles_of(w.n * p.group) - 1 - at;
    w.first = 0;
    w.last = blocks_seen(p, w.tile, w.n, w.len);
    return w;
}

// A number the compiler forgets what it is made of: what derives from it is computed where it is used, an instruction each, and
// kept in no register from block to block.
__device__ __forceinline__ uint32_t opaque(uint32_t x)
{
    asm volatile("" : "+v"(x));
    return x;
}
__device__ __forceinline__ int64_t opaque64(int64_t x)  // (the same for the wavefront)
{
    asm volatile("" : "+s"(x));
    return x;
}

// Tiles of all requests along a line, which is cut into ranges of the same length, one a workgroup, whatever tiles and parts
// of tiles they hold: all workgroups have as much to do.  (A sequence's first keys are seen by all its rows, twice the average.  Rows that
// are not shared go out longest first, which evens out many of them.)  Of rows: tile k of a request weighs what its last row sees,
// in units of 1/G key, and kPromptTileCost blocks more for what a tile costs by itself.  Of keys: what rows see its first key, in
// blocks of them.
enum { kLineRows, kLineKeys };
struct SharedLine {
    int32_t n[kMaxBatch], len[kMaxBatch], start[kMaxBatch];
    int64_t before[kMaxBatch];        // what the requests before weigh,
    int32_t tiles_before[kMaxBatch];  //   and their tiles
    int64_t wave[kWaves];
    int32_t tiles[kWaves], longest[kWaves];
};
struct Line {
    int64_t all, size;  // length of the line, and of a range
    int tiles;
    int start, n, len;  // of the only request, where there is one
    bool share;         // of rows: whether tiles are shared out, or each is one workgroup's
};
// What the tiles before a tile weigh together.
template <int KIND>
__device__ __forceinline__ int64_t weight_before(const PromptRows &p, int64_t tile, int n, int len)
{
    if (KIND == kLineRows)
        return tile * ((int64_t)p.group * (max(len - n, 0) + kPromptTileCost * kPromptKeys)) + kPromptRows / 2 * tile * (tile + 1);
    return tile * blocks_of(n * p.group) - (int64_t)(kPromptRows / kPromptKeys) * p.group * tile * (tile - 1) / 2;
}
template <int KIND>
__device__ __forceinline__ int line_tiles(const PromptRows &p, int n) { return tiles_of(KIND == kLineRows ? n * p.group : n); }

template <int KIND>
__device__ __forceinline__ Line lay_line(const PromptRows &p, double one_range, SharedLine &sh)
{
    const bool alone = p.batch == 1;  // (no LDS, no barrier)
    const int t = alone ? 0 : threadIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int start = 0, n = 0, len = 0;
    if (t < p.batch) request_of(p, t, start, n, len);
    Line l;
    l.start = start;
    l.n = n;
    l.len = len;
    l.tiles = line_tiles<KIND>(p, n);
    l.all = weight_before<KIND>(p, l.tiles, n, len);
    int longest = n > 0 ? blocks_of(len) : 0;
    if (!alone) {
        const int tiles = l.tiles;
        const int64_t weight = l.all;
        int tiles_upto = (int)wave_scan((uint32_t)tiles);
        int64_t upto = weight;
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t x = __shfl_up(upto, d);
            upto += lane >= d ? x : 0;
        }
        longest = (int)wave_max((uint32_t)longest);
        if (lane == 63) {
            sh.longest[wave] = longest;
            sh.tiles[wave] = tiles_upto;
            sh.wave[wave] = upto;
        }
        __syncthreads();
        l.tiles = 0;
        l.all = 0;
        longest = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            tiles_upto += i < wave ? sh.tiles[i] : 0;
            upto += i < wave ? sh.wave[i] : 0;
            l.tiles += sh.tiles[i];
            l.all += sh.wave[i];
            longest = max(longest, sh.longest[i]);
        }
        sh.n[t] = n;
        sh.len[t] = len;
        sh.start[t] = start;
        sh.before[t] = upto - weight;
        sh.tiles_before[t] = tiles_upto - tiles;
        __syncthreads();
    }
    const int unit = KIND == kLineRows ? p.group * kPromptKeys : 1;  // a block
    l.size = uniform64((int64_t)((double)l.all * one_range) + 1);
    l.size = uniform64(max(l.size, (int64_t)(KIND == kLineKeys ? kPromptMinKeyRange : kPromptMinRange) * unit));
    // A workgroup alone on its unit takes 1.2 us a block, one of two 2.05; a range costs its beginning, its partials and their merge.  One
    // prompt of 16 heads (4 KV heads), shared and not: 2048 tokens 43.5 us and 46, 3500 80 and 81, 5120 143 and 126, 6144 195 and 164;
    // of 4 heads (2) 1100 tokens 22 and 28, 2048 26 and 45, 8192 95 and 157.
    l.share = KIND == kLineKeys ||
              (float)__builtin_amdgcn_readfirstlane(longest) > kPromptShareCost + kPromptShareSize * (float)l.size / (float)unit;
    l.all = uniform64(l.all);
    l.tiles = __builtin_amdgcn_readfirstlane(l.tiles);
    l.start = __builtin_amdgcn_readfirstlane(l.start);
    l.n = __builtin_amdgcn_readfirstlane(l.n);
    l.len = __builtin_amdgcn_readfirstlane(l.len);
    return l;
}

struct LineTile {
    int b, tile, n, len, start;
    int number;          // among all requests' tiles
    int64_t at, weight;  // where the tile begins on the line, and what it weighs
};
// A request on the line: the tile's number is still the request's first one's, its place the request's.
__device__ __forceinline__ LineTile line_request(const PromptRows &p, int b, const Line &line, const SharedLine &sh)
{
    LineTile k;
    k.b = b;
    if (p.batch == 1) {
        k.n = line.n;
        k.len = line.len;
        k.start = line.start;
        k.number = 0;
        k.at = 0;
    } else {
        k.n = __builtin_amdgcn_readfirstlane(sh.n[b]);
        k.len = __builtin_amdgcn_readfirstlane(sh.len[b]);
        k.start = __builtin_amdgcn_readfirstlane(sh.start[b]);
        k.number = __builtin_amdgcn_readfirstlane(sh.tiles_before[b]);
        k.at = uniform64(sh.before[b]);
    }
    k.n = __builtin_amdgcn_readfirstlane(k.n);
    k.len = __builtin_amdgcn_readfirstlane(k.len);
    k.start = __builtin_amdgcn_readfirstlane(k.start);
    k.number = __builtin_amdgcn_readfirstlane(k.number);
    k.at = uniform64(k.at);
    return k;
}
// The tile that holds a place on the line.
template <int KIND>
__device__ __forceinline__ LineTile line_tile_at(const PromptRows &p, int64_t at, const Line &line, const SharedLine &sh)
{
    int b = 0;
    if (p.batch > 1)
        for (int step = kMaxBatch / 2; step > 0; step >>= 1)
            if (b + step < p.batch && uniform64(sh.before[b + step]) <= at) b += step;
    LineTile k = line_request(p, b, line, sh);
    const int tiles = line_tiles<KIND>(p, k.n);
    k.tile = 0;
    for (int step = tiles > 1 ? 1 << (31 - __builtin_clz(tiles - 1)) : 0; step > 0; step >>= 1)
        if (k.tile + step < tiles && weight_before<KIND>(p, k.tile + step, k.n, k.len) <= at - k.at) k.tile += step;
    const int64_t from = weight_before<KIND>(p, k.tile, k.n, k.len);
    k.weight = weight_before<KIND>(p, k.tile + 1, k.n, k.len) - from;
    k.at += from;
    k.number += k.tile;
    return k;
}
// Of a tile's blocks those before a place in it: 0 at its beginning, all at its end.  (In between an estimate: all that counts
// is that who asks for the same place gets the same answer, and for a later one no smaller.)
__device__ __forceinline__ int cut_at(int64_t place, int64_t weight, int blocks)
{
    const int cut = min((int)((float)place * ((float)blocks * __builtin_amdgcn_rcpf((float)weight))), blocks);
    return __builtin_amdgcn_readfirstlane(place <= 0 ? 0 : place >= weight ? blocks : cut);
}
// Which range holds a place on the line.
__device__ __forceinline__ int range_at(int64_t place, const Line &line)
{
    const int64_t size = opaque64(line.size);  // (so that its reciprocal is not kept through all the products)
    int64_t r = (int64_t)((double)place * __builtin_amdgcn_rcp((double)size));  // (one off at most)
    if (r * size > place) --r;
    if ((r + 1) * size <= place) ++r;
    return __builtin_amdgcn_readfirstlane((int)r);
}
// Partials: a range leaves two at most, that of the end of a tile that began in a range before, and that of a tile's beginning.
__device__ __forceinline__ int64_t part_slot(int64_t range, bool beginning, int n_kv_heads, int g)
{
    return (range * 2 + beginning) * n_kv_heads + g;
}
// For the merge, of a tile that lies in several ranges: how many (0: in one), the first of them, and what the tile is.  Kept by the range
// it begins in, which is the only one there, or, where there are fewer tiles, by its number.  (A launch's first microseconds
// go by the code that it runs once, which comes from memory: the merges read this, and lay no line.)
struct Record {
    int parts, range, tile, n, start, unused[3];
};
static_assert(sizeof(Record) == 4 * kRecordWords, "");
__device__ __forceinline__ void keep_record(int32_t *records, int at, const Record &r)
{
    typedef int i32x4_t __attribute__((ext_vector_type(4)));
    *(LYCHEE_GLOBAL i32x4_t *)(records + kRecordWords * at) = i32x4_t{r.parts, r.range, r.tile, r.n};
    gstore(records + kRecordWords * at + 4, r.start);
}
// What no tile will fill in; one workgroup's first threads.
__device__ __forceinline__ void clear_records(int32_t *records, int n_records, bool by_number, const Line &line, int range)
{
    if (by_number) {
        if (range == 0)
            for (int i = (line.share ? line.tiles : 0) + threadIdx.x; i < n_records; i += kThreads) gstore(records + kRecordWords * i, 0);
    } else if (threadIdx.x == 0 && range < n_records) {
        gstore(records + kRecordWords * range, 0);
    }
}
__device__ __forceinline__ void record_tile(int32_t *records, int n_records, bool by_number, const Line &line, const LineTile &k, int range,
                                            bool whole)
{
    const int at = by_number ? k.number : range;
    if (threadIdx.x == 0 && at < n_records && (by_number || !whole))
        keep_record(records, at, {whole ? 0 : range_at(k.at + k.weight - 1, line) - range + 1, range, k.tile, k.n, k.start, {}});
}
__device__ __forceinline__ Record recorded(const int32_t *records, int at)
{
    const int32_t *r = records + kRecordWords * at;
    const auto word = [&](int i) { return __builtin_amdgcn_readfirstlane(gload(r + i)); };
    return {word(0), word(1), word(2), word(3), word(4), {}};
}

// What a workgroup works on: where tiles are shared out a range of the line, tile after tile and parts of tiles at its ends; else one tile.
struct Work {
    Line line;
    bool share;
    int range;
    int64_t at, until;  // what is left of the range
    int slot;           // of the present tile's partials; -1: the workgroup has all of its blocks
    Tile w;
};
// (whether there is anything to do)
template <bool SHARE>
__device__ __forceinline__ bool begin_work(Work &k, const PromptRows &p, int g, double one_range, int32_t *records, int n_records,
                                           bool by_number, SharedLine &line, SharedPlan &plan)
{
    k.share = false;
    k.range = blockIdx.x / p.n_kv_heads;
    k.at = k.until = 0;
    k.slot = -1;
    if (SHARE) {
        k.line = lay_line<kLineRows>(p, one_range, line);
        k.share = k.line.share;
        k.at = k.range * k.line.size;
        k.until = k.share ? min(k.at + k.line.size, k.line.all) : 0;
        if (g == 0) clear_records(records, n_records, by_number, k.line, k.range);
        if (k.share) return k.at < k.until;
        __syncthreads();
    }
    k.w = find_tile(p, k.range, plan);
    return k.w.found;
}
// The next tile of a range, and which of its blocks.
__device__ __forceinline__ void next_tile(Work &k, const PromptRows &p, int g, int32_t *records, int n_records, bool by_number,
                                          const SharedLine &line)
{
    if (!k.share) return;
    const LineTile t = line_tile_at<kLineRows>(p, k.at, k.line, line);
    k.w = Tile{t.b, t.tile, t.n, t.len, t.start, 0, blocks_seen(p, t.tile, t.n, t.len), true};
    const int64_t from = k.at - t.at, to = min(opaque64(k.until) - t.at, t.weight);
    const int blocks = k.w.last;
    k.w.first = cut_at(from, t.weight, blocks);
    k.w.last = cut_at(to, t.weight, blocks);
    k.slot = from == 0 && to == t.weight ? -1 : (int)part_slot(k.range, from == 0, p.n_kv_heads, g);
    if (from == 0 && g == 0) record_tile(records, n_records, by_number, k.line, t, k.range, to == t.weight);
    k.at += to - from;
}
__device__ __forceinline__ bool more_work(const Work &k) { return k.share && k.at < opaque64(k.until); }

// ------------------------------------------------------------------------------ LDS
// Sixteen bytes a lane from global memory to LDS, lane after lane from `to` on (base and to: the same for the wavefront).  In
// assembly, because the compiler lets every later read of LDS wait for such a copy at once, whichever part of LDS it writes; the
// kernels wait themselves, before the barrier behind which the copied block is read.
template <typename T>
__device__ __forceinline__ const T *uniform(const T *p)  // (in scalar registers, whatever the compiler knows of it)
{
    const uint64_t u = reinterpret_cast<uint64_t>(p);
    const uint32_t high = (uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32));
    return reinterpret_cast<const T *>((uint64_t)high << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)u));
}
__device__ __forceinline__ void copy16(const uint16_t *base, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void copy4(const float *base, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
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
    const s16x4_t b =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((LYCHEE_LDS s16x4_t *)(p + 8 * kRowBytes + (place ^ (uint32_t)(db << 6 | 32))));
    typedef short s16x8_t __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8_t, (s16x8_t)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
// Nothing is moved over this: reads of LDS stay as far ahead of the products that need them as they are written.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }
// Waits for loads of the compiler's own here.  It does not see that wait_copies() waits for them too, and would wait for them at their
// first use in the loop, every turn: by then that is a wait for the copies just begun.
template <int N>
__device__ __forceinline__ void arrived(bf16x8_t (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        u32x4_t bits = __builtin_bit_cast(u32x4_t, x[i]);
        asm volatile("" : "+v"(bits));
        x[i] = __builtin_bit_cast(bf16x8_t, bits);
    }
}

// Pairs that must not count have a weight of zero, but zero times an infinity or NaN is NaN.  A workgroup whose sums hold
// no numbers makes them again with care, every block three times: with zeros for such values (turn 0), and then with finite numbers
// that put them back where they count.  The largest bf16 number, squared, is an infinity in fp32: turn 1 has it, with its
// sign, for infinities and NaN, the products' other operand being that number for the pairs that count and zero for the others
// (seen_rows), and turn 2 its negative for NaN, which both infinities add up to.  The block is changed in LDS, where it
// makes scores too behind the products that do.
constexpr uint32_t kLargest = 0x7F7Fu;
__device__ __forceinline__ void take_with_care(uint8_t *block, int bytes, int turn)
{
#pragma unroll 1
    for (int i = (int)opaque(threadIdx.x); i < bytes / 4; i += kThreads) {
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
// The pairs that count, of step s in the order of read_turned: rows least .. most of the block's.  Weights that are not positive, dS of an
// infinite key, are 0 or no number, and make NaN of its infinities: turn 1 twice, the second time with `largest` negative.
__device__ __forceinline__ bf16x8_t seen_rows(int hi, int s, int least, int most, uint32_t largest = kLargest)
{
    u32x4_t u;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int row = 16 * s + 4 * hi + (w & 1) * 2 + (w >> 1) * 8;
        u[w] = (row >= least && row <= most ? largest : 0u) | (row + 1 >= least && row + 1 <= most ? largest << 16 : 0u);
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

// Whether any thread of the workgroup says so.
__device__ __forceinline__ bool any_thread(bool x, int wave, int (&said)[kWaves])
{
    const bool any = __ballot(x) != 0;
    __syncthreads();  // (the last answer has been read)
    said[wave] = any;
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(said[0] | said[1] | said[2] | said[3]) != 0;
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

// A wavefront's sums as a partial, in the order of the registers: 1 KB a store, read back alike.
__device__ __forceinline__ void store_part(float *to, const f32x16_t (&x)[4])
{
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x4_t y = {x[db][4 * j], x[db][4 * j + 1], x[db][4 * j + 2], x[db][4 * j + 3]};
            *(LYCHEE_GLOBAL f32x4_t *)(to + (4 * db + j) * 256) = y;
        }
}
// Four neighbouring dimensions of a merged row.
__device__ __forceinline__ void store_four(uint16_t *to, f32x4_t x, float f)
{
    *(LYCHEE_GLOBAL u32x2_t *)to = u32x2_t{pk_bf16(x[0] * f, x[1] * f), pk_bf16(x[2] * f, x[3] * f)};
}

}  // namespace
}  // namespace lychee
