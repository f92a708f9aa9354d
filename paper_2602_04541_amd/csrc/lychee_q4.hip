// The paged 4-bit cache: writing it, reading it back, and decode attention over it.  The layout is lychee.h's: tiles of
// 16 tokens of one KV head, a token's key and value side by side in one 128-byte line, the tile's scales in a
// seventeenth line.  A gathered token therefore costs one line and one line of scales, and a streamed sequence is
// contiguous tile by tile.
#include "lychee_device.h"
#include "lychee_paged.h"

namespace lychee {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;

// Orders what the lanes of a wavefront hand to one another through LDS (whose accesses a wavefront makes in order).
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// The cache is read once a step: nontemporal loads.
__device__ __forceinline__ uint4 load16(const uint8_t *p) { return load_stream16(reinterpret_cast<const uint16_t *>(p)); }
__device__ __forceinline__ int clamp_tokens(int L, int most) { return L < 0 ? 0 : (L > most ? most : L); }

// ------------------------------------------------------------------------------ append
// Magnitudes of two bf16 numbers, ordered as 16-bit integers (a NaN's is the largest).
__device__ __forceinline__ uint32_t pk_max_u16(uint32_t a, uint32_t b)
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// The scale byte of a group whose largest magnitude has these bf16 bits: the smallest e with m <= 6 * 2^e.  With
// m = (1 + f/128) * 2^(E-127): 6 * 2^e >= m first holds for e = E-129 if f <= 64 (m <= 1.5 * 2^(E-127)), else E-128.
__device__ __forceinline__ uint32_t scale_byte(uint32_t m)
{
    const int E = (int)(m >> 7), f = (int)(m & 0x7F);
    if (E == 255) return 255u;  // a NaN or an infinity
    const int s = E - 2 + (f > 64);
    return (uint32_t)(s < kScaleMin ? kScaleMin : (s > kScaleMax ? kScaleMax : s));
}

// Eight bf16 numbers as codes.
__device__ __forceinline__ uint32_t codes8(uint4 x, uint32_t s)
{
    const float scale = __builtin_bit_cast(float, s << 23);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.x), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.y), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.z), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.w), scale, 3);
    return s == 255u ? 0u : c;
}

// Largest magnitude of a group: 8 numbers a lane, 4 lanes.
__device__ __forceinline__ uint32_t group_max(uint4 x)
{
    const uint32_t m = 0x7FFF7FFFu;
    uint32_t a = pk_max_u16(pk_max_u16(x.x & m, x.y & m), pk_max_u16(x.z & m, x.w & m));
    a = pk_max_u16(a, dpp_u32<0xB1>(a));  // lane ^ 1
    a = pk_max_u16(a, dpp_u32<0x4E>(a));  // lane ^ 2
    return max(a & 0xFFFFu, a >> 16);
}

// 16 lanes a (token, head): 16 bytes of key and of value each.  Bound by memory: 70.7K tokens of 8 heads, 366 MB, in 64.8 us
// (5.7 TB/s).  A workgroup has 16 tokens of one head, since tokens that follow one another mostly share a tile, and the scale
// bytes of a wavefront's four then go to one line (four heads of a token a wavefront: 69 us, 60 without the scales).
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a)
{
    const uint32_t H = (uint32_t)a.d.n_kv_heads, g = blockIdx.x % H;
    const int i = (int)(blockIdx.x / H) * (kThreads / 16) + (int)(threadIdx.x >> 4);
    const int lane = threadIdx.x & 15;
    if (i >= a.n_tokens) return;  // (whole groups of 16 lanes)
    const int slot = gload(a.slots + i);
    const int64_t from = (int64_t)i * a.stride_tok + (int64_t)g * a.stride_head + 8 * lane;
    const uint4 k = load_stream16(a.k_new + from), v = load_stream16(a.v_new + from);
    const uint32_t ks = scale_byte(group_max(k)), vs = scale_byte(group_max(v));
    const int page = slot >> a.d.page_shift, off = slot & ((1 << a.d.page_shift) - 1);
    if (slot < 0 || page >= a.d.n_pages) return;
    const int sub = off & (kTileTokens - 1);
    uint8_t *tile = a.cache +
                    ((int64_t)page * a.d.page_tiles + (int64_t)g * ((1 << a.d.page_shift) / kTileTokens) + off / kTileTokens) * kTileBytes;
    uint32_t *to = reinterpret_cast<uint32_t *>(tile + sub * kTokenBytes);
    gstore(to + lane, codes8(k, ks));
    gstore(to + 16 + lane, codes8(v, vs));
    if ((lane & 3) == 0) {
        uint8_t *sc = tile + kTileScales + (lane >> 2) * kTileTokens + sub;
        gstore(sc, (uint8_t)ks);
        gstore(sc + 4 * kTileTokens, (uint8_t)vs);
    }
}

// ------------------------------------------------------------------------------ read
// Byte i as the scale of a conversion, which reads a float's exponent field alone (what the neighbouring bytes leave in
// the sign and the mantissa is ignored).
__device__ __forceinline__ float scale_of(uint32_t bytes, int i)
{
    return __builtin_bit_cast(float, i == 0 ? bytes << 23 : i == 1 ? bytes << 15 : i == 2 ? bytes << 7 : bytes >> 1);
}

// Eight codes as bf16 numbers, exactly: e2m1 times a power of two, within bf16's normal range for every scale byte that
// append writes; 255 makes them NaN.
__device__ __forceinline__ uint4 decode8(uint32_t c, float scale)
{
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3)));
}
// 16 lanes a row: a dword of key and of value each, 16 bytes of either out.  Bound by memory, four fifths of it writes: 2.4 GB
// in 415 us, 5.7 TB/s (a copy of 1 GiB reaches 5.0).  Nontemporal stores, since nobody here reads the rows again (453 us with
// the others), and one row a group of lanes (two rows 437, four 453).
__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a)
{
    const int g = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 15;
    const int first = a.first ? clamp_tokens(gload(a.first + b), a.d.max_len) : 0;
    const int last = clamp_tokens(gload(a.last + b), a.d.max_len);
    const int r = blockIdx.x * (kThreads / 16) + (int)(threadIdx.x >> 4);
    if (r >= min(a.n_rows, last - first)) return;
    const int t = first + r;
    const int page = gload(a.table + (int64_t)b * a.d.table_stride + (t >> a.d.page_shift));
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    if ((uint32_t)page < (uint32_t)a.d.n_pages) {
        const int off = t & ((1 << a.d.page_shift) - 1), sub = off & (kTileTokens - 1);
        const uint8_t *tile = a.cache + ((int64_t)page * a.d.page_tiles + (int64_t)g * ((1 << a.d.page_shift) / kTileTokens) +
                                         off / kTileTokens) * kTileBytes;
        const uint32_t *row = reinterpret_cast<const uint32_t *>(tile + sub * kTokenBytes);
        const uint8_t *sc = tile + kTileScales + (lane >> 2) * kTileTokens + sub;
        k = decode8(gload(row + lane), scale_of(gload(sc), 0));
        v = decode8(gload(row + 16 + lane), scale_of(gload(sc + 4 * kTileTokens), 0));
    }
    const int64_t to = (int64_t)b * a.stride_b + (int64_t)g * a.stride_h + (int64_t)r * a.stride_t + 8 * lane;
    __builtin_nontemporal_store(u32x4_t{k.x, k.y, k.z, k.w}, (LYCHEE_GLOBAL u32x4_t *)(a.k_out + to));
    __builtin_nontemporal_store(u32x4_t{v.x, v.y, v.z, v.w}, (LYCHEE_GLOBAL u32x4_t *)(a.v_out + to));
}

// ------------------------------------------------------------------------------ attention
// One query token a request: for the query heads h of a KV head's group
//     s_h[t] = q_h . K[t] / sqrt(128),  m = max s,  l = sum 2^(s - m),  o = sum 2^(s - m) V[t] / l     (log2 units)
// in one pass over the tokens with a running m and l.
//
// The space of work is blocks of 64 tokens of a segment, a segment being a (request, KV head, kind of head): its whole
// sequence for retrieval heads, its set for sparse ones.  Segments are cut into pieces (split_size), and a workgroup takes
// one piece after another; in a piece each of its four wavefronts takes every fourth block with an (m, l, o) of its own.
// They are merged in LDS when the piece ends; a piece that is a whole segment writes the output, others leave a partial,
// and the workgroup that completes a segment merges its partials.
//
// What bounds it: 131072 tokens of 8 KV heads (142.6 MB) take 33.6 us (35.2 over several caches in turn, none of which the
// last-level cache holds), of which the loop has 23 (loads alone 19, 7.1 TB/s; arithmetic alone 12, for four query heads a KV
// head), the start 5 (the cut, page entries, the first lines 2 us away) and the merge of the partials 5.  64 short requests
// (109 MB, 15 us of reading) take 29.3 us, which is their longest one's, in one piece: a wavefront takes 2 to 2.7 us for each
// block of 64 tokens, being a chain through LDS and the matrix units that two wavefronts a SIMD hide only in part.  Groups of
// 9 to 16 query heads have twice the products, and up to 16 heads' partials that one workgroup merges: 32768 tokens of two such
// KV heads (8.9 MB) take 33 us.  Two workgroups a CU: three need 168 registers, and spill (a fifth slower).
//
// A wavefront's block of 64 tokens is four tiles (of a set: four times 16 rows of it), which go from the cache to registers in
// whole lines, 16 bytes a lane (loaded in the pieces that the lanes need instead, 16 and 4 bytes of many rows, a 128K layer
// took 37 us without any arithmetic), one block ahead, and through LDS to the lanes that need them.  Rows lie 144 bytes
// apart there and tiles 2624, so that 16 lanes read 16 rows, and four rows of lanes four tokens, from banks of their own.
// Lane (g, n) = (lane / 16, lane % 16); position 4n + a of the block is token 16a + n:
//   scores  v_mfma_f32_16x16x32_bf16, A = queries (16 rows), B = the keys of tile a (column n: row n), 4 times along the
//           dimensions.  Head number i of the segment is row 4(i%4) + i/4, so that lane (g, n) has the scores of heads g,
//           g+4, .. in its registers 0, 1, ..: with the usual four heads every lane works on one number in the softmax.
//           A lane takes 16 bytes of a key, its dimensions 32g .. 32g+31 under one scale byte, and converts them (two
//           numbers an instruction, exactly); which dimension is which in the sum does not matter as long as the
//           queries are laid out alike.
//   weights go to LDS in order of position as bf16, hi + lo, off by 2^-17 of a weight at most: of one in [2^e, 2^(e+1))
//           hi leaves up to 2^(e-8), and half a place of that in bf16 is 2^(e-17).  One bf16 number would be off by 2^-8, as
//           much as the output's own rounding, and the matrix units' fp32 products run at a sixteenth of bf16's rate.  The
//           sum l has the weights unrounded.  Rows that the heads leave free hold lo, so that with up to 8 heads the two
//           products cost one.  They come back as the A operand of the second product: lane (g, row) gets positions 16g + 8s .. + 7
//           in step s of 2.
//   values  lane (g, n) takes dword n (dimensions 8n .. 8n+7) of the values of those tokens, converts them and pairs
//           neighbouring positions (v_perm): the B operands of eight products, product d giving dimension 8n + d.  A
//           scale is applied where it belongs, to the numbers of its token and group.
constexpr int kRowPad = kTokenBytes + 16;            // from one row to the next in LDS
constexpr int kTilePad = 2624;                       // and from one tile to the next: 16 rows, 128 bytes of scales, 192 unused
constexpr int kScalesAt = kTileTokens * kRowPad;
static_assert(kScalesAt + 128 <= kTilePad && kTilePad % 256 == 64, "four tiles' rows of one number in banks of their own");

struct Block {
    uint4 row[8];    // lane: 16 bytes, number lane % 8, of rows 8j + lane / 8
    uint4 scale;     // streaming: 16 bytes, number lane % 8, of the scales of tile lane / 8
    uint8_t sc[8];   // gathering: the scale bytes of token `lane`
    uint64_t bad;    // tokens that are not there, one bit each
};

constexpr int kPRow = 144;  // bytes from one row of weights in LDS to the next (64 x 2, and off the same banks)
template <int R>
struct SharedQ4 {
    __align__(16) int32_t len[kMaxBatch];
    float pieces[kWaves][kSplits];   // of the sizes of a piece that are weighed
    uint32_t classes[kWaves][kSplits];
    uint8_t order[kMaxBatch];        // requests, the longest first
    uint16_t rmask[kMaxKvHeads];
    uint8_t rhead[kMaxKvHeads], ghead[kMaxKvHeads];
    int32_t heads[kQ4MaxGroup];      // query heads of the piece's segment
    int32_t last;
    __align__(16) uint8_t p[kWaves][(R == 4 ? 2 : 1) * 16 * kPRow];  // weights; rows that no head writes stay zero
    __align__(16) uint32_t row[kWaves][kQ4Block];                    // gathered tokens: tile * 16 + place
    union {
        __align__(16) uint8_t tile[kWaves][4 * kTilePad];
        struct {
            __align__(16) float o[kWaves][4 * R][kHeadDim];
            float ml[kWaves][4 * R][2];
        } red;
        struct {
            float w[4 * R][kQ4MaxWg];
            float l[4 * R];
            __align__(16) float o[kThreads / 32][4][kHeadDim];
        } comb;
    };
};

__device__ __forceinline__ float max16(float x)  // over the 16 lanes of a row
{
    x = fmaxf(x, dpp_f32<0xB1>(x));
    x = fmaxf(x, dpp_f32<0x4E>(x));
    x = fmaxf(x, dpp_f32<0x141>(x));
    x = fmaxf(x, dpp_f32<0x140>(x));
    return x;
}

__device__ __forceinline__ uint32_t pk_bf16(float a, float b)  // round to nearest even, a in the low half
{
    bf16x2_t r;
    r[0] = (__bf16)a;
    r[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, r);
}

__device__ __forceinline__ bf16x8_t as_frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_bit_cast(bf16x8_t, u32x4_t{a, b, c, d});
}
// The part of a segment a wavefront works on, and where its tokens are.
struct Seq {
    const int32_t *table;  // the request's row of the block table
    const int32_t *set;    // entries of the set (GATHER)
    const uint8_t *cache;
    int32_t len;           // tokens of the request
    int32_t n;             // tokens (entries) of the segment
    int32_t last;          // the set's last entry
    int32_t head_tile;     // first tile of the KV head within a page
};

template <int R, bool GATHER, bool SCORES>
struct Piece {
    // Streaming: page entries of 16 of the wavefront's blocks, four tiles each, one a lane (block i's tile x in lane 4i + x).
    static __device__ __forceinline__ int fetch_entries(const Q4AttnArgs &a, const Seq &s, int lane, int blk, int end)
    {
        const int most = max(0, (s.n - 1) / kTileTokens);
        const int tile = min(min(blk + kWaves * (lane >> 2), end - 1) * 4 + (lane & 3), most);
        return gload(s.table + (tile >> (a.d.page_shift - 4)));
    }
    static __device__ __forceinline__ int fetch_index(const Seq &s, int lane, int blk)
    {
        const int e = blk * kQ4Block + lane;
        const int at = gload(s.set + min(e, s.last));
        return e < s.n && (uint32_t)at < (uint32_t)s.len ? at : -1;
    }
    static __device__ __forceinline__ int fetch_page(const Q4AttnArgs &a, const Seq &s, int at)
    {
        return gload(s.table + (max(at, 0) >> a.d.page_shift));
    }

    // Loads a streamed block; entries: of fetch_entries, i: which of its blocks.  Tiles that are not there are read as some
    // tile that is.
    static __device__ __forceinline__ void stream(const Q4AttnArgs &a, const Seq &s, int lane, int blk, int entries, int i, Block &t)
    {
        const int ps = a.d.page_shift, tiles = 1 << (ps - 4);
        const uint8_t *base[4];
        t.bad = 0;
        if (ps >= 6) {  // (the same for the launch) a block lies in one page, all of it addressable
            const int page = __builtin_amdgcn_readlane(entries, 4 * i);
            const bool bad = (uint32_t)page >= (uint32_t)a.d.n_pages;
            t.bad = bad ? ~0ull : 0ull;
            base[0] = s.cache + ((int64_t)(bad ? 0 : page) * a.d.page_tiles + s.head_tile + ((blk * 4) & (tiles - 1))) * kTileBytes;
#pragma unroll
            for (int x = 1; x < 4; ++x) base[x] = base[0] + x * kTileBytes;
        } else {
            const int most = max(0, (s.n - 1) / kTileTokens);  // the last tile
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int page = __builtin_amdgcn_readlane(entries, 4 * i + x);
                const bool bad = (uint32_t)page >= (uint32_t)a.d.n_pages;
                t.bad |= bad ? 0xFFFFull << (16 * x) : 0ull;
                base[x] = s.cache + ((int64_t)(bad ? 0 : page) * a.d.page_tiles + s.head_tile + (min(blk * 4 + x, most) & (tiles - 1))) * kTileBytes;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) t.row[j] = load16(base[j >> 1] + (uint32_t)((j & 1) * 1024 + 16 * lane));
        const int x = (lane >> 3) & 3;
        const uint8_t *sb = x < 2 ? (x == 0 ? base[0] : base[1]) : (x == 2 ? base[2] : base[3]);
        t.scale = load16(sb + kTileScales + 16 * (lane & 7));
    }

    // The same for a block of a set: `at` and `page` are this lane's token and its page.
    static __device__ __forceinline__ void gather(const Q4AttnArgs &a, const Seq &s, int lane, int at, int page, Block &t, uint32_t *rows)
    {
        const int ps = a.d.page_shift;
        const bool ok = at >= 0 && (uint32_t)page < (uint32_t)a.d.n_pages;
        const int off = max(at, 0) & ((1 << ps) - 1);
        const uint32_t row = ((uint32_t)(ok ? page : 0) * (uint32_t)a.d.page_tiles + (uint32_t)s.head_tile + (uint32_t)(off >> 4)) * 16u + (off & 15);
        t.bad = __ballot(!ok);
        rows[lane] = row;
        wave_sync();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t r = rows[8 * j + (lane >> 3)];
            t.row[j] = load16(s.cache + (int64_t)(r + (r >> 4)) * kTokenBytes + 16 * (lane & 7));
        }
        const uint8_t *sc = s.cache + (int64_t)(row >> 4) * kTileBytes + kTileScales + (row & 15);
#pragma unroll
        for (int i = 0; i < 8; ++i) t.sc[i] = gload(sc + i * kTileTokens);
        wave_sync();
    }

    // A loaded block into the wavefront's tiles in LDS.
    static __device__ __forceinline__ void stage(const Block &t, int lane, uint8_t *tile)
    {
        uint8_t *to = tile + (lane >> 3) * kRowPad + 16 * (lane & 7);
#pragma unroll
        for (int j = 0; j < 8; ++j) *reinterpret_cast<uint4 *>(to + (j >> 1) * kTilePad + (j & 1) * 8 * kRowPad) = t.row[j];
        if (GATHER) {
            uint8_t *sc = tile + (lane >> 4) * kTilePad + kScalesAt + (lane & 15);
#pragma unroll
            for (int i = 0; i < 8; ++i) sc[i * kTileTokens] = t.sc[i];
        } else if (lane < 32) {
            *reinterpret_cast<uint4 *>(tile + (lane >> 3) * kTilePad + kScalesAt + 16 * (lane & 7)) = t.scale;
        }
        wave_sync();
    }

    // Scores, weights and weighted values of a staged block; bad: of its Block.
    static __device__ __forceinline__ void consume(const Q4AttnArgs &a, const Seq &s, int lane, int blk, uint64_t bad, const uint8_t *tile,
                                                   const bf16x8_t (&qf)[4], float (&m)[R], float (&l)[R], f32x4_t (&o)[8], uint8_t *p,
                                                   float *scores, float pool_scale)
    {
        const int n = lane & 15, g = lane >> 4;
        f32x4_t z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            z[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            const float sc = scale_of(tile[i * kTilePad + kScalesAt + g * kTileTokens + n], 0);
            const uint4 k = *reinterpret_cast<const uint4 *>(tile + i * kTilePad + n * kRowPad + 16 * g);
            const uint32_t kd[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint4 x = decode8(kd[c], sc);
                z[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[c], as_frag(x.x, x.y, x.z, x.w), z[i], 0, 0, 0);
            }
            if (i & 1) __builtin_amdgcn_sched_barrier(0);  // (else all four tiles' conversions are made at once, and spilled)
        }
        uint32_t vs[4];  // scale bytes of values: tile i, tokens 4g .. 4g+3
#pragma unroll
        for (int i = 0; i < 4; ++i)
            vs[i] = *reinterpret_cast<const uint32_t *>(tile + i * kTilePad + kScalesAt + (4 + (n >> 2)) * kTileTokens + 4 * g);
        // Tokens that do not count (behind a segment's last, or without a page): their scores are -infinity, and the scales
        // of their values 2^-127, a number, since a weight of 0 times NaN is NaN.
        if (!GATHER && (blk + 1) * kQ4Block > s.n) bad |= s.n <= blk * kQ4Block ? ~0ull : ~0ull << (s.n - blk * kQ4Block);
        if (bad != 0) {
            asm volatile("");  // (a branch: these are many instructions, and rare)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t b = (uint32_t)(bad >> (16 * i)) & 0xFFFFu;
#pragma unroll
                for (int r = 0; r < R; ++r) z[i][r] = (b >> n) & 1u ? -__builtin_inff() : z[i][r];
#pragma unroll
                for (int j = 0; j < 4; ++j) vs[i] &= (b >> (4 * g + j)) & 1u ? ~(0xFFu << (8 * j)) : ~0u;
            }
        }
        if (SCORES) {
            float sum[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[i] = z[i][0];
#pragma unroll
                for (int r = 1; r < R; ++r) sum[i] += z[i][r];
            }
            // (over the four rows of lanes: row g ends with the sums of tile g, lane by lane)
            const float x = sum_halves32_pair(sum_rows16_pair(sum[0], sum[1]), sum_rows16_pair(sum[2], sum[3]));
            const int at = blk * kQ4Block + lane;
            if (at < s.n) gstore(scores + at, x * pool_scale);
        }
        float w[4][R];
        bool raise = false;
        float top[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i][r] = z[i][r] * a.scale_log2e;
            }
            top[r] = max16(fmaxf(fmaxf(w[0][r], w[1][r]), fmaxf(w[2][r], w[3][r])));
            raise |= top[r] > m[r];
        }
        if (__ballot(raise) != 0) {  // (the same for all the lanes of a head; rescaling is rare after the first blocks)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float up = fmaxf(m[r], top[r]);
                const float f = m[r] == up ? 1.0f : fast_exp2(m[r] - up);  // (-inf - finite: 0)
                m[r] = up;
                l[r] *= f;
#pragma unroll
                for (int d = 0; d < 8; ++d) {
                    o[d][r] *= f;
                    if (R <= 2) o[d][R + r] *= f;
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float base = m[r] == -__builtin_inff() ? 0.0f : m[r];
            float lo[4];
            uint32_t hi[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i][r] = fast_exp2(w[i][r] - base);
                l[r] += w[i][r];
            }
            hi[0] = pk_bf16(w[0][r], w[1][r]);
            hi[1] = pk_bf16(w[2][r], w[3][r]);
            lo[0] = w[0][r] - bf16_lo(hi[0]);
            lo[1] = w[1][r] - bf16_hi(hi[0]);
            lo[2] = w[2][r] - bf16_lo(hi[1]);
            lo[3] = w[3][r] - bf16_hi(hi[1]);
            *reinterpret_cast<uint2 *>(p + (4 * g + r) * kPRow + 8 * n) = make_uint2(hi[0], hi[1]);
            *reinterpret_cast<uint2 *>(p + (R <= 2 ? 4 * g + R + r : 16 + 4 * g + r) * kPRow + 8 * n) =
                make_uint2(pk_bf16(lo[0], lo[1]), pk_bf16(lo[2], lo[3]));
        }
        wave_sync();
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const bf16x8_t pf = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t *>(p + n * kPRow + 32 * g + 16 * st));
            bf16x8_t pl;
            if (R == 4) pl = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t *>(p + (16 + n) * kPRow + 32 * g + 16 * st));
            float sc[8];
            uint32_t v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {  // position 16g + 8st + j: tile j % 4, row 4g + 2st + j / 4
                sc[j] = scale_of(vs[j & 3], 2 * st + (j >> 2));
                v[j] = *reinterpret_cast<const uint32_t *>(tile + (j & 3) * kTilePad + (4 * g + 2 * st + (j >> 2)) * kRowPad + 64 + 4 * n);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t c[8], even[4], odd[4];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t x = v[j];
                    c[j] = __builtin_bit_cast(uint32_t, i == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, sc[j], 0)
                                                        : i == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, sc[j], 1)
                                                        : i == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, sc[j], 2)
                                                                 : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, sc[j], 3));
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    even[j] = __builtin_amdgcn_perm(c[2 * j + 1], c[2 * j], 0x05040100u);
                    odd[j] = __builtin_amdgcn_perm(c[2 * j + 1], c[2 * j], 0x07060302u);
                }
                const bf16x8_t ve = as_frag(even[0], even[1], even[2], even[3]), vo = as_frag(odd[0], odd[1], odd[2], odd[3]);
                o[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf, ve, o[2 * i], 0, 0, 0);
                o[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf, vo, o[2 * i + 1], 0, 0, 0);
                if (R == 4) {
                    o[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pl, ve, o[2 * i], 0, 0, 0);
                    o[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pl, vo, o[2 * i + 1], 0, 0, 0);
                }
                if (i & 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
        wave_sync();
    }

    // Blocks [b0, b0 + nb) of a segment with `heads` heads (sh.heads).  slot < 0: the piece is the whole segment and writes the
    // output; else its partial goes to that slot.
    static __device__ __forceinline__ void run(const Q4AttnArgs &a, const Seq &s, int b, int g0, int heads, int b0, int nb, int64_t slot,
                                               SharedQ4<R> &sh)
    {
        const int tid = fresh_tid(), lane = tid & 63, wave = uni(tid >> 6), n = lane & 15, g = lane >> 4;
        const int end = b0 + nb;
        int blk = b0 + wave;
        int entries = 0, at = 0, at2 = 0, page = 0;
        if (GATHER) {
            at = fetch_index(s, lane, min(blk, end - 1));
            at2 = fetch_index(s, lane, min(blk + kWaves, end - 1));
        } else {
            entries = fetch_entries(a, s, lane, min(blk, end - 1), end);
        }
        bf16x8_t qf[4];
        {
            // head number i is row 4 (i % 4) + i / 4: row n is head number (n / 4) + 4 (n % 4)
            const int h = (n >> 2) + 4 * (n & 3);
            const bool mine = (n & 3) < R && h < heads;
            const uint16_t *q = a.q + ((int64_t)b * a.d.n_kv_heads * a.d.group + (int64_t)g0 * a.d.group + (mine ? sh.heads[h] : 0)) * kHeadDim + 32 * g;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint4 x = gload_u4(q + 8 * c);
                qf[c] = mine ? as_frag(x.x, x.y, x.z, x.w) : as_frag(0, 0, 0, 0);
            }
        }
        float m[R], l[R];
        f32x4_t o[8];
#pragma unroll
        for (int r = 0; r < R; ++r) m[r] = -__builtin_inff(), l[r] = 0.0f;
#pragma unroll
        for (int d = 0; d < 8; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        uint8_t *p = sh.p[wave];
        float *scores = SCORES ? a.scores + ((int64_t)b * a.d.n_kv_heads + g0) * a.score_stride : nullptr;
        const float pool_scale = a.scale / (float)heads;
        if (blk < end) {
            // One block is in flight while another is worked on; what its addresses need is loaded earlier: 16 blocks' page
            // entries at a time, or a set's entries two blocks and their pages one block before the rows.
            Block t;
            uint32_t *rows = sh.row[wave];
            uint8_t *tile = sh.tile[wave];
            int next_entries = entries, done = 0;
            if (GATHER) page = fetch_page(a, s, at);
            auto fetch = [&](Block &t, int blk) {  // (blocks in order; behind the last one again and again)
                if (GATHER) {
                    const int at_now = at, page_now = page;
                    at = at2;
                    page = fetch_page(a, s, at);
                    at2 = fetch_index(s, lane, min(blk + 2 * kWaves, end - 1));
                    gather(a, s, lane, at_now, page_now, t, rows);
                } else {
                    stream(a, s, lane, min(blk, end - 1), entries, done & 15, t);
                    ++done;
                    if ((done & 15) == 8) next_entries = fetch_entries(a, s, lane, blk + 9 * kWaves, end);  // (of blocks 16, 17, ..)
                    if ((done & 15) == 0) entries = next_entries;
                }
            };
            auto step = [&]() {
                stage(t, lane, tile);
                const uint64_t bad = t.bad;
                fetch(t, blk + kWaves);
                consume(a, s, lane, blk, bad, tile, qf, m, l, o, p, scores, pool_scale);
                blk += kWaves;
                return blk < end;
            };
            fetch(t, blk);
            while (step()) {
            }
        }
        __syncthreads();  // (the weights' rows become the sums')
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float sum = row16_sum(l[r]);
            const int h = g + 4 * r;
            float *to = &sh.red.o[wave][h][8 * n];
            float4 x, y;
            x.x = o[0][r], x.y = o[1][r], x.z = o[2][r], x.w = o[3][r];
            y.x = o[4][r], y.y = o[5][r], y.z = o[6][r], y.w = o[7][r];
            if (R <= 2) {
                x.x += o[0][(R + r) & 3], x.y += o[1][(R + r) & 3], x.z += o[2][(R + r) & 3], x.w += o[3][(R + r) & 3];
                y.x += o[4][(R + r) & 3], y.y += o[5][(R + r) & 3], y.z += o[6][(R + r) & 3], y.w += o[7][(R + r) & 3];
            }
            reinterpret_cast<float4 *>(to)[0] = x;
            reinterpret_cast<float4 *>(to)[1] = y;
            if (n == 0) {
                sh.red.ml[wave][h][0] = m[r];
                sh.red.ml[wave][h][1] = sum;
            }
        }
        __syncthreads();
        for (int e = tid; e < heads * kHeadDim; e += kThreads) {
            const int h = e / kHeadDim, d = e % kHeadDim;
            float M = sh.red.ml[0][h][0];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sh.red.ml[w][h][0]);
            const float base = M == -__builtin_inff() ? 0.0f : M;
            float sum = 0.0f, x = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = fast_exp2(sh.red.ml[w][h][0] - base);
                sum = fmaf(f, sh.red.ml[w][h][1], sum);
                x = fmaf(f, sh.red.o[w][h][d], x);
            }
            if (slot < 0) {
                const int64_t row = ((int64_t)b * a.d.n_kv_heads + g0) * a.d.group + sh.heads[h];
                gstore(a.out + row * kHeadDim + d, f32_to_bf16(sum == 0.0f ? 0.0f : x / sum));
            } else {
                gstore_through(a.part_o + (slot * a.d.group + h) * kHeadDim + d, x);
                if (d < 2) gstore_through(a.part_ml + (slot * a.d.group + h) * 2 + d, d == 0 ? M : sum);
            }
        }
        if (slot >= 0) wait_stores();
        __syncthreads();
    }

    static __device__ __forceinline__ uint16_t f32_to_bf16(float x)
    {
        return __builtin_bit_cast(uint16_t, (__bf16)x);  // (a NaN stays one)
    }
};

// Merges the partials of a segment, slots s0 .. s0 + count - 1, into the output.  The weights of a head's slots are one
// wavefront's; 32 lanes have the columns of a head, four each, and eight groups of them share its slots, of four heads at a
// time.  The partials come from memory, 2 us away: the first ones are asked for before the weights are known, and up to 64
// slots of up to four heads all at once.
template <int R>
__device__ __forceinline__ void merge(const Q4AttnArgs &a, int b, int g0, int heads, int64_t s0, int count, SharedQ4<R> &sh)
{
    const int tid = fresh_tid(), lane = tid & 63, wave = tid >> 6, c4 = tid & 31, grp = tid >> 5;
    constexpr int kGroups = kThreads / 32;
    const char *po = reinterpret_cast<const char *>(uni(a.part_o + s0 * a.d.group * kHeadDim));  // (32-bit offsets from here)
    const char *pm = reinterpret_cast<const char *>(uni(a.part_ml + s0 * a.d.group * 2));
    auto part = [&](int i, int h) {
        return gload_f4(reinterpret_cast<const float *>(po + (uint32_t)((min(i, count - 1) * a.d.group + min(h, heads - 1)) * kHeadDim * 4 + 16 * c4)));
    };
    auto weigh = [&]() {
        for (int h = wave; h < heads; h += kWaves) {
            float M = -__builtin_inff(), l = 0.0f;
            for (int i = lane; i < count; i += 64)
                M = fmaxf(M, gload_f2(reinterpret_cast<const float *>(pm + (uint32_t)((i * a.d.group + h) * 8))).x);
            M = wave_max_f(M);
            const float base = M == -__builtin_inff() ? 0.0f : M;
            for (int i = lane; i < count; i += 64) {
                const float2 ml = gload_f2(reinterpret_cast<const float *>(pm + (uint32_t)((i * a.d.group + h) * 8)));
                const float f = fast_exp2(ml.x - base);
                sh.comb.w[h][i] = f;
                l = fmaf(f, ml.y, l);
            }
            l = sum_halves32(sum_rows16(row16_sum(l)));
            if (lane == 0) sh.comb.l[h] = l;
        }
        __syncthreads();
    };
    float4 acc[4];
    auto add = [&](int i, int h0, const float4 (&v)[4]) {
        if (i >= count) return;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const float w = sh.comb.w[min(h0 + h, heads - 1)][i];
            acc[h].x = fmaf(w, v[h].x, acc[h].x);
            acc[h].y = fmaf(w, v[h].y, acc[h].y);
            acc[h].z = fmaf(w, v[h].z, acc[h].z);
            acc[h].w = fmaf(w, v[h].w, acc[h].w);
        }
    };
    auto clear = [&]() {
#pragma unroll
        for (int h = 0; h < 4; ++h) acc[h] = make_float4(0.f, 0.f, 0.f, 0.f);
    };
    auto finish = [&](int h0) {
#pragma unroll
        for (int h = 0; h < 4; ++h) reinterpret_cast<float4 *>(sh.comb.o[grp][h])[c4] = acc[h];
        __syncthreads();
        for (int e = tid; e < min(4, heads - h0) * kHeadDim; e += kThreads) {
            const int h = e / kHeadDim, d = e % kHeadDim;
            float x = 0.0f;
#pragma unroll
            for (int i = 0; i < kGroups; ++i) x += sh.comb.o[i][h][d];
            const float l = sh.comb.l[h0 + h];
            const int64_t row = ((int64_t)b * a.d.n_kv_heads + g0) * a.d.group + sh.heads[h0 + h];
            gstore(a.out + row * kHeadDim + d, __builtin_bit_cast(uint16_t, (__bf16)(l == 0.0f ? 0.0f : x / l)));
        }
        __syncthreads();
    };
    if (count <= 8 * kGroups && heads <= 4) {
        float4 v[8][4];
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
            for (int h = 0; h < 4; ++h) v[u][h] = part(grp + u * kGroups, h);
        weigh();
        clear();
#pragma unroll
        for (int u = 0; u < 8; ++u) add(grp + u * kGroups, 0, v[u]);
        finish(0);
        return;
    }
    weigh();
#pragma unroll 1
    for (int h0 = 0; h0 < heads; h0 += 4) {
        clear();
#pragma unroll 1
        for (int i0 = grp; i0 < count; i0 += 4 * kGroups) {
            float4 v[4][4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int h = 0; h < 4; ++h) v[u][h] = part(i0 + u * kGroups, h0 + h);
#pragma unroll
            for (int u = 0; u < 4; ++u) add(i0 + u * kGroups, h0, v[u]);
        }
        finish(h0);
    }
}

// How a launch is cut into pieces.  A piece costs as much as kPieceCost blocks whatever its length (its chain of loads, its
// merge in LDS, its partial: 5 us, in which four wavefronts take 8 to 10 blocks; 6, 9, 12 and 16 blocks give the same times
// within their noise on the 16 shapes below), and one that is not a whole segment makes another workgroup merge partials.  So
// segments are cut into pieces of at most `size` blocks, for the size of kSplits candidates that is cheapest: the longest piece
// counts, or where there are more pieces than workgroups, the mean of what a workgroup has and what cutting adds, if that is
// more.  What it adds (kCutCost a piece) is no cost that was measured but a weight that was fitted: 160 against 12 takes 64
// requests of 61 to 3001 tokens from 36 to 31 us, 48 of 1000 to 6000 from 52 to 48, 100 of 100 to 8000 from 82 to 79, 128 of
// 100 to 4000 from 62 to 63, and changes nothing on 12 shapes more.  The mean does not see that workgroups take whole
// pieces, and no size is below an equal share: 65 requests of 20000 tokens of 8 KV heads are 520 segments, which are not cut, and
// take 315 us where 64 take 216 (of 3000 tokens 57 and 40).  Sizes start at an equal share of all blocks, four at least, and
// are multiples of four, a block for each wavefront.
// Piece number i is workgroup i's; of more pieces than workgroups, the next ones go to the workgroups in turn, forwards and
// backwards (claimed from a counter they took as long).  Numbers go by the kind of head, retrieval first, since sets are
// mostly the shorter segments, and within it from the longest to the shortest request: a launch's workgroups begin over some
// 5 us, in order, and two share a CU.  64 requests of 61 to 3001 tokens 37 -> 31 us, 256 of up to 2000 27 -> 25, 200 over sets
// 41 -> 36, and by the kind of head 8 of 16K to 96K over sets of 2048 55.7 -> 53.6, over 4096 44.4 -> 42.3.
// Requests are ordered by length where workgroups take several pieces or the batch is larger than 16.  Finding the order costs
// 0.5 to 1 us (2 to 16 requests whose pieces all fit: 16.3 -> 17.1, 12.5 -> 13.3, 19.3 -> 20.2 with it); without it 60 requests
// of 61 to 3001 tokens in 480 pieces take 36 us instead of 29.  Large batches of few pieces, which need it least, pay for that:
// 40 requests on 2 KV heads 17 -> 18 us, 200 of up to 2000 tokens 23 -> 26.
__device__ __forceinline__ int split_size(int share, int c)  // candidate c: 1, 9/8, .. 15/8, 2, 3, 4, 6, 8, 16, 64 shares, whole segments
{
    if (c == kSplits - 1) return 1 << 28;
    const int eighths = c < 8 ? 8 + c : c == 8 ? 16 : c == 9 ? 24 : c == 10 ? 32 : c == 11 ? 48 : c == 12 ? 64 : c == 13 ? 128 : 512;
    return (int)((((int64_t)share * eighths + 31) / 32) * 4);
}
// Pieces of a segment of n blocks, and how many blocks each has (the last may have fewer).
__device__ __forceinline__ int piece_blocks(int n, int size)
{
    if (size >= n) return n;
    const int pieces = quot(n + size - 1, size);
    return quot(n + pieces - 1, pieces);
}
__device__ __forceinline__ int piece_count(int n, int size)
{
    const int each = piece_blocks(n, size);
    return quot(n + each - 1, each);
}

__device__ __forceinline__ int wave_sum(int x)
{
    return (int)__builtin_amdgcn_readlane((int)wave_scan((uint32_t)x), 63);
}

template <int R, bool SETS, bool SCORES>
__global__ __launch_bounds__(kThreads, 2) void q4_attn_kernel(Q4AttnArgs a)
{
    __shared__ SharedQ4<R> sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), B = a.d.batch, H = a.d.n_kv_heads;
    // Every wavefront works out the whole cut for itself: lane i has requests i * each .. i * each + each - 1.  (Loops that
    // are not unrolled: a launch's instructions come from memory, and most have one request a lane.)
    const int each = (B + 63) >> 6;
    sh.rmask[lane] = a.rmask[lane];  // (here and below: every wavefront writes the same, and needs no barrier)
    sh.rhead[lane] = a.rhead[lane];
    sh.ghead[lane] = a.ghead[lane];
    static_assert(kMaxKvHeads == 64, "a lane each");
    for (int i = lane; i < (int)sizeof sh.p[0] / 16; i += 64) reinterpret_cast<uint4 *>(sh.p[wave])[i] = make_uint4(0, 0, 0, 0);
    // (an empty segment is one block of tokens that do not count: its outputs are zero like any other's)
    auto blocks_of = [&](int n) { return max(1, (n + kQ4Block - 1) / kQ4Block); };
    auto set_blocks = [&](int n) { return blocks_of(min(n, a.d.k)); };
    const int first = lane * each, last = min(first + each, B);
    int blocks = 0, most_tokens = 0;
#pragma unroll 1
    for (int r = first; r < last; ++r) {
        const int L = clamp_tokens(gload(a.lengths + r), a.d.max_len);
        most_tokens = max(most_tokens, L);
        sh.len[r] = L;  // (by every wavefront, the same)
        blocks += a.n_rseg * blocks_of(L) + (SETS ? a.n_gseg * set_blocks(L) : 0);
    }
    const int T = wave_sum(blocks);
    most_tokens = (int)wave_max((uint32_t)most_tokens);
    const int share = max(kWaves, quot_uni(T + a.n_wg - 1, a.n_wg));
    const float inv_wg = __builtin_amdgcn_rcpf((float)a.n_wg);
    wave_sync();
    // Lane (g, c): candidate c and every fourth request; in a large batch the wavefronts share the requests as well.
    const bool shared = B > 16;
    const int mine_of = split_size(share, lane & (kSplits - 1)), some = min(mine_of, 1 << 20);
    const float inv = __builtin_amdgcn_rcpf((float)some);
    int sum = 0;
#pragma unroll 1
    for (int r = shared ? 4 * wave + (lane >> 4) : lane >> 4; r < B; r += shared ? 4 * kWaves : 4) {
        const int L = sh.len[r];
        sum += a.n_rseg * quot_by(blocks_of(L) + some - 1, some, inv, [](uint32_t v) { return v; });
        if (SETS) sum += a.n_gseg * quot_by(set_blocks(L) + some - 1, some, inv, [](uint32_t v) { return v; });
    }
    float pieces = sum_halves32(sum_rows16((float)sum));  // (far fewer than 2^24)
    if (shared) {
        sh.pieces[wave][lane & (kSplits - 1)] = pieces;
        __syncthreads();
        pieces = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) pieces += sh.pieces[w][lane & (kSplits - 1)];
    }
    const float longest = (float)min(some, SETS && a.n_rseg == 0 ? set_blocks(most_tokens) : blocks_of(most_tokens));
    const float cut = (pieces - (float)(B * (a.n_rseg + (SETS ? a.n_gseg : 0)))) * kCutCost;
    const float cost = fmaxf(kPieceCost + longest, pieces <= (float)a.n_wg ? 0.0f : (pieces * kPieceCost + cut + (float)T) * inv_wg + 0.5f * kPieceCost);
    const float least = -wave_max_f(-cost);
    const int size = uni(split_size(share, (int)__builtin_ctzll(__ballot(cost == least))));
    // Pieces of the lane's requests, of retrieval and of sparse heads, and with those of the lanes before.
    int r_mine, g_mine, r_upto, g_upto;
    auto count_pieces = [&](auto request) {
        r_mine = g_mine = g_upto = 0;
#pragma unroll 1
        for (int r = first; r < last; ++r) {
            const int L = sh.len[request(r)];
            r_mine += a.n_rseg * piece_count(blocks_of(L), size);
            if (SETS) g_mine += a.n_gseg * piece_count(set_blocks(L), size);
        }
        r_upto = (int)wave_scan((uint32_t)r_mine);
        if (SETS) g_upto = (int)wave_scan((uint32_t)g_mine);
    };
    count_pieces([](int r) { return r; });
    const int n_r = __builtin_amdgcn_readlane(r_upto, 63), N = n_r + __builtin_amdgcn_readlane(g_upto, 63);
    // The longest requests first (in 16 classes, else as they are numbered), so that what begins late is short: thread r finds
    // the place of request r.
    const bool ordered = B > 16 || N > a.n_wg;
    if (ordered) {
        const float part = 15.99f * __builtin_amdgcn_rcpf((float)max(1, most_tokens));
        const int cls = tid < B ? max(0, 15 - (int)((float)sh.len[tid] * part)) : kSplits;
        unsigned long long same = 0;
        uint32_t count = 0;
#pragma unroll
        for (int c = 0; c < kSplits; ++c) {
            const unsigned long long m = __ballot(cls == c);
            same = cls == c ? m : same;
            count = lane == c ? (uint32_t)__builtin_popcountll(m) : count;
        }
        if (lane < kSplits) sh.classes[wave][lane] = count;
        __syncthreads();
        const uint32_t x = sh.classes[lane & 3][lane >> 2];
        const int before = __shfl((int)(wave_scan(x) - x), (cls & (kSplits - 1)) * 4 + wave);
        if (tid < B) sh.order[before + __builtin_popcountll(same & ((1ull << lane) - 1ull))] = (uint8_t)tid;
        __syncthreads();
        count_pieces([&](int r) { return (int)sh.order[r]; });
    }
    for (int round = 0, at = blockIdx.x; at < N; ++round, at = round * a.n_wg + (round & 1 ? a.n_wg - 1 - (int)blockIdx.x : (int)blockIdx.x)) {
        // the kind of head, request, KV head and part that piece `at` is
        const bool gather = SETS && at >= n_r;
        const int nth = gather ? at - n_r : at, upto = gather ? g_upto : r_upto;
        const int who = (int)__builtin_popcountll(__ballot(upto <= nth));
        int rel = nth - __builtin_amdgcn_readlane(upto - (gather ? g_mine : r_mine), who), place = who * each, b, L, per, parts;
#pragma unroll 1
        for (;; ++place) {
            b = ordered ? uni((int)sh.order[place]) : place;
            L = uni(sh.len[b]);
            per = gather ? set_blocks(L) : blocks_of(L);
            parts = uni(piece_count(per, size));
            const int all = parts * (gather ? a.n_gseg : a.n_rseg);
            if (rel < all) break;
            rel -= all;
        }
        const int si = uni(quot(rel, parts)), part = rel - si * parts;
        const int most = uni(piece_blocks(per, size));
        const int j = part * most, nb = min(most, per - j);
        const int g = uni((int)(gather ? sh.ghead[si] : sh.rhead[si]));
        uint32_t heads_mask = uni((uint32_t)sh.rmask[g]);
        if (gather) heads_mask = ~heads_mask & ((1u << a.d.group) - 1u);
        const int heads = __builtin_popcount(heads_mask);
        if (tid < kQ4MaxGroup && ((heads_mask >> tid) & 1u)) sh.heads[__builtin_popcount(heads_mask & ((1u << tid) - 1u))] = tid;
        __syncthreads();
        Seq s;
        s.table = a.table + (int64_t)b * a.d.table_stride;
        s.set = SETS ? a.idx_in + ((int64_t)b * H + g) * a.d.k : nullptr;
        s.cache = a.cache;
        s.len = L;
        s.n = gather ? min(L, a.d.k) : L;
        s.last = a.d.k - 1;
        s.head_tile = g << (a.d.page_shift - 4);
        const int64_t slot = parts == 1 ? -1 : at;  // (a partial's slot is the piece's number)
        if (SETS && gather) Piece<R, true, false>::run(a, s, b, g, heads, j, nb, slot, sh);
        else Piece<R, false, SCORES>::run(a, s, b, g, heads, j, nb, slot, sh);
        if (tid == 0) {
            int last = 0;
            if (parts > 1) {
                uint32_t *counter = a.seg_count + (((int64_t)b * H + g) * 2 + (gather ? 1 : 0)) * kLineWords;
                const uint32_t old = __hip_atomic_fetch_add((LYCHEE_GLOBAL uint32_t *)counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                last = old + 1 == (uint32_t)parts;
                if (last) gstore_through(counter, 0u);  // as every launch finds it
            }
            sh.last = last;
        }
        __syncthreads();
        if (sh.last) {
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
            merge<R>(a, b, g, heads, at - part, parts, sh);
        }
        __syncthreads();
    }
}

template <int R>
hipError_t launch_r(const Q4AttnArgs &a, hipStream_t stream)
{
    if (a.n_gseg == 0) {
        if (a.scores == nullptr) q4_attn_kernel<R, false, false><<<a.n_wg, kThreads, 0, stream>>>(a);
        else q4_attn_kernel<R, false, true><<<a.n_wg, kThreads, 0, stream>>>(a);
    } else {
        if (a.scores == nullptr) q4_attn_kernel<R, true, false><<<a.n_wg, kThreads, 0, stream>>>(a);
        else q4_attn_kernel<R, true, true><<<a.n_wg, kThreads, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, hipStream_t stream)
{
    const int64_t groups = (a.n_tokens + kThreads / 16 - 1) / (kThreads / 16);
    append_kernel<<<(uint32_t)(groups * a.d.n_kv_heads), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_read(const ReadArgs &a, hipStream_t stream)
{
    const dim3 grid((uint32_t)((a.n_rows + kThreads / 16 - 1) / (kThreads / 16)), (uint32_t)a.d.n_kv_heads, (uint32_t)a.d.batch);
    read_kernel<<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

// A launch is one build, by the shape's group, whatever the head types divide it into: R numbers of every lane's softmax are
// 4R heads.  Wider than needed costs: a group of 4 at 128K takes 32.1 us with R = 1, 33.0 with 2, 36.1 with 4; a group of 8 (64
// short requests) 31.3 with 2, 36 with 4.
hipError_t launch_q4_attn(const Q4AttnArgs &a, hipStream_t stream)
{
    return a.d.group <= 4 ? launch_r<1>(a, stream) : a.d.group <= 8 ? launch_r<2>(a, stream) : launch_r<4>(a, stream);
}

}  // namespace lychee
