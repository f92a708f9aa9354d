// The paged 4-bit cache: writing it, reading it back, and decode attention over it.  The layout is lychee.h's: tiles of
// 16 tokens of one KV head, a token's key and value side by side in one 128-byte line, the tile's scales in a
// seventeenth line.  A gathered token therefore costs one line and one line of scales, and a streamed sequence is
// contiguous tile by tile.
#include "lychee_device.h"
#include "lychee_paged.h"

namespace lychee {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;

__device__ __forceinline__ int clamp_tokens(int L, int most) { return L < 0 ? 0 : (L > most ? most : L); }
__device__ __forceinline__ int64_t tile_at(int32_t tile) { return (int64_t)tile * kTileBytes; }

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

// 16 lanes a (token, head): 16 bytes of key and of value each.
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a)
{
    const int64_t row = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
    const int lane = threadIdx.x & 15;
    const uint32_t H = (uint32_t)a.d.n_kv_heads;
    if (row >= (int64_t)a.n_tokens * H) return;  // (whole groups of 16 lanes)
    const uint32_t i = (uint32_t)(row / H), g = (uint32_t)(row - (int64_t)i * H);
    const int slot = gload(a.slots + i);
    const int64_t from = (int64_t)i * a.stride_tok + (int64_t)g * a.stride_head + 8 * lane;
    const uint4 k = load_stream16(a.k_new + from), v = load_stream16(a.v_new + from);
    const uint32_t ks = scale_byte(group_max(k)), vs = scale_byte(group_max(v));
    const int page = slot >> a.d.page_shift, off = slot & ((1 << a.d.page_shift) - 1);
    if (slot < 0 || page >= a.d.n_pages) return;
    const int sub = off & (kTileTokens - 1);
    uint8_t *tile = a.cache + tile_at(0) +
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
// Eight codes as bf16 numbers, exactly: e2m1 times a power of two, within bf16's normal range for every scale byte that
// append writes; 255 makes them NaN.
__device__ __forceinline__ uint4 decode8(uint32_t c, uint32_t s)
{
    const float scale = __builtin_bit_cast(float, s << 23);
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3)));
}
__device__ __forceinline__ void gstore_u4(uint16_t *p, uint4 v) { *(LYCHEE_GLOBAL u32x4_t *)p = u32x4_t{v.x, v.y, v.z, v.w}; }

constexpr int kReadRows = 64;  // rows of a (request, head) a workgroup takes
// 16 lanes a row: a dword of key and of value each, 16 bytes of either out.
__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a)
{
    const int g = blockIdx.y, b = blockIdx.z;
    const int first = a.first ? clamp_tokens(gload(a.first + b), a.d.max_len) : 0;
    const int last = clamp_tokens(gload(a.last + b), a.d.max_len);
    const int lane = threadIdx.x & 15;
    const int n = min(a.n_rows, last - first);
#pragma unroll
    for (int u = 0; u < kReadRows / (kThreads / 16); ++u) {
        const int r = blockIdx.x * kReadRows + u * (kThreads / 16) + (int)(threadIdx.x >> 4);
        if (r >= n) return;
        const int t = first + r;
        const int page = gload(a.table + (int64_t)b * a.d.table_stride + (t >> a.d.page_shift));
        uint4 k = make_uint4(0, 0, 0, 0), v = k;
        if ((uint32_t)page < (uint32_t)a.d.n_pages) {
            const int off = t & ((1 << a.d.page_shift) - 1), sub = off & (kTileTokens - 1);
            const uint8_t *tile = a.cache + ((int64_t)page * a.d.page_tiles + (int64_t)g * ((1 << a.d.page_shift) / kTileTokens) +
                                             off / kTileTokens) * kTileBytes;
            const uint32_t *row = reinterpret_cast<const uint32_t *>(tile + sub * kTokenBytes);
            const uint8_t *sc = tile + kTileScales + (lane >> 2) * kTileTokens + sub;
            k = decode8(gload(row + lane), gload(sc));
            v = decode8(gload(row + 16 + lane), gload(sc + 4 * kTileTokens));
        }
        const int64_t to = (int64_t)b * a.stride_b + (int64_t)g * a.stride_h + (int64_t)r * a.stride_t + 8 * lane;
        gstore_u4(a.k_out + to, k);
        gstore_u4(a.v_out + to, v);
    }
}

// ------------------------------------------------------------------------------ attention
// One query token a request: for the query heads h of a KV head's group
//     s_h[t] = q_h . K[t] / sqrt(128),  m = max s,  l = sum 2^(s - m),  o = sum 2^(s - m) V[t] / l     (log2 units)
// in one pass over the tokens with a running m and l.
//
// The space of work is blocks of 64 tokens of a segment, a segment being a (request, KV head, kind of head): its whole
// sequence for retrieval heads, its set for sparse ones.  A workgroup takes a contiguous run of blocks, cut into pieces
// where segments end; in a piece each of its four wavefronts takes every fourth block with an (m, l, o) of its own.
// They are merged in LDS when the piece ends; a piece that is a whole segment writes the output, others leave a partial,
// and the workgroup that completes a segment merges its partials.
//
// A wavefront's block: lane (g, n) = (lane / 16, lane % 16).
//   scores  v_mfma_f32_16x16x32_bf16, A = queries (16 rows), B = keys (16 tokens), 4 times along the dimensions, for 4
//           groups of 16 tokens: group a's column n is token 4n + a.  Head number i of the segment is row 4(i%4) + i/4,
//           so that lane (g, n) has the scores of heads g, g+4, .. in its registers 0, 1, ..: with the usual four heads
//           every lane works on one number in the softmax.  A lane loads 16 bytes of a key, its dimensions 32g .. 32g+31
//           under one scale byte, straight from the cache, and converts them (two numbers an instruction, exactly);
//           which dimension is which in the sum does not matter as long as the queries are laid out alike.
//   weights go to LDS as bf16, hi + lo (rows that the heads leave free hold lo: the two products cost one), and come
//           back as the A operand of the second product: lane (g, row) gets tokens 16g + 8s .. + 7 in step s of 2.
//   values  lane (g, n) loads dword n (dimensions 8n .. 8n+7) of the values of tokens 16g .. 16g+15 and their scale bytes
//           as one 16-byte load, converts them and pairs neighbouring tokens (v_perm): the B operands of eight products,
//           product d giving dimension 8n + d.  So values are never transposed through LDS, and a scale is applied
//           where it belongs, to the numbers of its token and group.
struct Tile4 {
    uint4 k[4];       // rows of tokens 4n .. 4n+3, dimensions 32g ..
    uint32_t v[16];   // dword n of the values of tokens 16g .. 16g+15
    uint32_t ks;      // scale bytes of the keys
    uint4 vs;         // and of the values
    int bad;          // not 0: some token of the block does not count
};

constexpr int kPRow = 144;  // bytes from one row of weights in LDS to the next (64 x 2, and off the same banks)
template <int R>
struct SharedQ4 {
    int32_t pre[kMaxBatch + 1];      // blocks of the requests before
    int32_t len[kMaxBatch];
    uint32_t scan[kWaves + 1];
    uint16_t rmask[kMaxKvHeads];
    uint8_t rhead[kMaxKvHeads], ghead[kMaxKvHeads];
    int32_t heads[kQ4MaxGroup];      // query heads of the piece's segment
    int32_t last;
    union {
        struct {
            __align__(16) uint8_t p[kWaves][(R == 4 ? 2 : 1) * 16 * kPRow];
            __align__(16) uint32_t row[kWaves][kQ4Block];       // gathered tokens: tile * 16 + place, ~0 = none
            __align__(16) uint8_t scale[kWaves][8 * kQ4Block];  // and their scale bytes
        };
        struct {
            __align__(16) float o[kWaves][4 * R][kHeadDim];
            float ml[kWaves][4 * R][2];
        } red;
        struct {
            float w[4 * R][kQ4MaxWg];
            float l[4 * R];
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
__device__ __forceinline__ float scale_of(uint32_t bytes, int i)
{
    const uint32_t s = i == 0 ? bytes << 23 : i == 1 ? bytes << 15 : i == 2 ? bytes << 7 : bytes >> 1;
    return __builtin_bit_cast(float, s & 0x7F800000u);
}

// The part of a segment a wavefront works on, and where its tokens are.
struct Seq {
    const int32_t *table;  // the request's row of the block table
    const int32_t *set;    // entries of the set (GATHER)
    const uint8_t *cache;
    int32_t len;           // tokens of the request
    int32_t n;             // tokens (entries) of the segment
    int32_t head_tile;     // first tile of the KV head within a page
};

template <int R, bool GATHER, bool SCORES>
struct Piece {
    // Loads a block's tokens.  Addresses of tokens that do not count are those of some that are there.
    static __device__ __forceinline__ void fetch(const Q4AttnArgs &a, const Seq &s, int blk, Tile4 &t, uint32_t *rows, uint8_t *scales)
    {
        const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
        const int ps = a.d.page_shift, tiles = 1 << (ps - 4);
        if (!GATHER) {
            const int most = max(0, (s.n - 1) / kTileTokens);  // the last tile
            const int kt = min(blk * 4 + (n >> 2), most), vt = min(blk * 4 + g, most);
            int kp = gload(s.table + (kt >> (ps - 4))), vp = gload(s.table + (vt >> (ps - 4)));
            const bool k_bad = (uint32_t)kp >= (uint32_t)a.d.n_pages, v_bad = (uint32_t)vp >= (uint32_t)a.d.n_pages;
            t.bad = (k_bad ? 1 : 0) | (v_bad ? 2 : 0);
            kp = k_bad ? 0 : kp;
            vp = v_bad ? 0 : vp;
            const uint8_t *kb = s.cache + ((int64_t)kp * a.d.page_tiles + s.head_tile + (kt & (tiles - 1))) * kTileBytes;
            const uint8_t *vb = s.cache + ((int64_t)vp * a.d.page_tiles + s.head_tile + (vt & (tiles - 1))) * kTileBytes;
#pragma unroll
            for (int i = 0; i < 4; ++i) t.k[i] = gload_u4(kb + (4 * (n & 3) + i) * kTokenBytes + 16 * g);
            t.ks = gload(reinterpret_cast<const uint32_t *>(kb + kTileScales + g * kTileTokens + 4 * (n & 3)));
#pragma unroll
            for (int j = 0; j < 16; ++j) t.v[j] = gload(reinterpret_cast<const uint32_t *>(vb + j * kTokenBytes + 64 + 4 * n));
            t.vs = gload_u4(vb + kTileScales + (4 + (n >> 2)) * kTileTokens);
        } else {
            const int e = blk * kQ4Block + lane;
            const int at = e < s.n ? gload(s.set + e) : -1;
            const bool in = (uint32_t)at < (uint32_t)s.len;
            const int tok = in ? at : 0;
            int page = gload(s.table + (tok >> ps));
            const bool ok = in && (uint32_t)page < (uint32_t)a.d.n_pages;
            page = ok ? page : 0;
            const int off = tok & ((1 << ps) - 1);
            const uint32_t row = ((uint32_t)page * (uint32_t)a.d.page_tiles + (uint32_t)s.head_tile + (uint32_t)(off >> 4)) * 16u + (off & 15);
            t.bad = !ok;
            rows[lane] = row;
            const uint8_t *sc = s.cache + (int64_t)(row >> 4) * kTileBytes + kTileScales + (row & 15);
#pragma unroll
            for (int i = 0; i < 8; ++i) scales[i * kQ4Block + lane] = ok ? gload(sc + i * kTileTokens) : (uint8_t)127;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            const uint4 kr = *reinterpret_cast<const uint4 *>(rows + 4 * n);
            const uint32_t krow[4] = {kr.x, kr.y, kr.z, kr.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) t.k[i] = gload_u4(s.cache + (int64_t)(krow[i] + (krow[i] >> 4)) * 128 + 16 * g);
            t.ks = *reinterpret_cast<const uint32_t *>(scales + g * kQ4Block + 4 * n);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint4 vr = *reinterpret_cast<const uint4 *>(rows + 16 * g + 4 * q);
                const uint32_t vrow[4] = {vr.x, vr.y, vr.z, vr.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    t.v[4 * q + i] = gload(reinterpret_cast<const uint32_t *>(s.cache + (int64_t)(vrow[i] + (vrow[i] >> 4)) * 128 + 64 + 4 * n));
            }
            t.vs = *reinterpret_cast<const uint4 *>(scales + (4 + (n >> 2)) * kQ4Block + 16 * g);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }

    // Scores, weights and weighted values of a block.
    static __device__ __forceinline__ void consume(const Q4AttnArgs &a, const Seq &s, int blk, Tile4 &t, const bf16x8_t (&qf)[4],
                                                   float (&m)[R], float (&l)[R], f32x4_t (&o)[8], uint8_t *p, float *scores,
                                                   float pool_scale)
    {
        const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
        f32x4_t z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            z[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            const float sc = scale_of(t.ks, i);
            const uint32_t kd[4] = {t.k[i].x, t.k[i].y, t.k[i].z, t.k[i].w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                bf16x8_t kf;
                const auto k0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kd[c], sc, 0);
                const auto k1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kd[c], sc, 1);
                const auto k2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kd[c], sc, 2);
                const auto k3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kd[c], sc, 3);
                kf = as_frag(__builtin_bit_cast(uint32_t, k0), __builtin_bit_cast(uint32_t, k1), __builtin_bit_cast(uint32_t, k2),
                             __builtin_bit_cast(uint32_t, k3));
                z[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[c], kf, z[i], 0, 0, 0);
            }
        }
        // which of the lane's four tokens count (all but in a segment's last block, and where pages are missing)
        const bool part = !GATHER && (blk + 1) * kQ4Block > s.n;
        uint32_t out_of = 0;  // bit i: token 4n + i does not count
        uint32_t v_out = 0;   // bit j: value 16g + j does not
        const unsigned long long any = __ballot(t.bad != 0);
        const bool ragged = part || any != 0;
        if (ragged) {
            if (GATHER) {
                out_of = (uint32_t)(any >> (4 * n)) & 15u;
                v_out = (uint32_t)(any >> (16 * g)) & 0xFFFFu;
            } else {
                const int k0 = blk * kQ4Block + 4 * n, v0 = blk * kQ4Block + 16 * g;
#pragma unroll
                for (int i = 0; i < 4; ++i) out_of |= (k0 + i >= s.n || (t.bad & 1)) ? 1u << i : 0u;
#pragma unroll
                for (int j = 0; j < 16; ++j) v_out |= (v0 + j >= s.n || (t.bad & 2)) ? 1u << j : 0u;
            }
        }
        if (SCORES) {
            float sum[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[i] = z[i][0];
#pragma unroll
                for (int r = 1; r < R; ++r) sum[i] += z[i][r];
                if (ragged && ((out_of >> i) & 1u)) sum[i] = -__builtin_inff();
            }
            // (over the four rows of lanes: row g ends with the sums of tokens 4n + g)
            const float x = sum_halves32_pair(sum_rows16_pair(sum[0], sum[1]), sum_rows16_pair(sum[2], sum[3]));
            const int at = blk * kQ4Block + 4 * n + g;
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
                if (ragged && ((out_of >> i) & 1u)) w[i][r] = -__builtin_inff();
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
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        uint32_t vs[4] = {t.vs.x, t.vs.y, t.vs.z, t.vs.w};
        if (ragged) {  // a value that does not count has weight 0: make its scale a number
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if ((v_out >> j) & 1u) vs[j >> 2] &= ~(0xFFu << (8 * (j & 3)));
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const bf16x8_t pf = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t *>(p + n * kPRow + 32 * g + 16 * st));
            bf16x8_t pl;
            if (R == 4) pl = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t *>(p + (16 + n) * kPRow + 32 * g + 16 * st));
            float sc[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) sc[j] = scale_of(vs[2 * st + (j >> 2)], j & 3);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t c[8], even[4], odd[4];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t x = t.v[8 * st + j];
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
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }

    // Blocks [b0, b0 + nb) of a segment with `heads` heads (sh.heads).  slot < 0: the piece is the whole segment and writes the
    // output; else its partial goes to that slot.
    static __device__ __forceinline__ void run(const Q4AttnArgs &a, const Seq &s, int b, int g0, int heads, int b0, int nb, int64_t slot,
                                               SharedQ4<R> &sh)
    {
        const int tid = fresh_tid(), lane = tid & 63, wave = uni(tid >> 6), n = lane & 15, g = lane >> 4;
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
        // (rows of weights that no head writes stay zero)
        for (int i = lane; i < (int)sizeof sh.p[0] / 16; i += 64) reinterpret_cast<uint4 *>(p)[i] = make_uint4(0, 0, 0, 0);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        float *scores = SCORES ? a.scores + ((int64_t)b * a.d.n_kv_heads + g0) * a.score_stride : nullptr;
        const float pool_scale = a.scale / (float)heads;
        const int end = b0 + nb;
        int blk = b0 + wave;
        if (blk < end) {
            Tile4 t0, t1;
            fetch(a, s, blk, t0, sh.row[wave], sh.scale[wave]);
            for (;;) {
                fetch(a, s, min(blk + kWaves, end - 1), t1, sh.row[wave], sh.scale[wave]);
                consume(a, s, blk, t0, qf, m, l, o, p, scores, pool_scale);
                blk += kWaves;
                if (blk >= end) break;
                fetch(a, s, min(blk + kWaves, end - 1), t0, sh.row[wave], sh.scale[wave]);
                consume(a, s, blk, t1, qf, m, l, o, p, scores, pool_scale);
                blk += kWaves;
                if (blk >= end) break;
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

// Merges the partials of a segment, slots s0 .. s0 + count - 1, into the output.
template <int R>
__device__ __forceinline__ void merge(const Q4AttnArgs &a, int b, int g0, int heads, int64_t s0, int count, SharedQ4<R> &sh)
{
    const int tid = fresh_tid(), lane = tid & 63, wave = tid >> 6;
    for (int h = wave; h < heads; h += kWaves) {
        float M = -__builtin_inff();
        for (int i = lane; i < count; i += 64) {
            const float m = gload_f2(a.part_ml + ((s0 + i) * a.d.group + h) * 2).x;
            sh.comb.w[h][i] = m;
            M = fmaxf(M, m);
        }
        M = wave_max_f(M);
        const float base = M == -__builtin_inff() ? 0.0f : M;
        float l = 0.0f;
        for (int i = lane; i < count; i += 64) {
            const float f = fast_exp2(sh.comb.w[h][i] - base);
            l = fmaf(f, gload_f2(a.part_ml + ((s0 + i) * a.d.group + h) * 2).y, l);
            sh.comb.w[h][i] = f;
        }
        l = sum_halves32(sum_rows16(row16_sum(l)));
        if (lane == 0) sh.comb.l[h] = l;
    }
    __syncthreads();
    for (int e = tid; e < heads * kHeadDim; e += kThreads) {
        const int h = e / kHeadDim, d = e % kHeadDim;
        const float *from = a.part_o + (s0 * a.d.group + h) * kHeadDim + d;
        float x = 0.0f;
#pragma unroll 16
        for (int i = 0; i < count; ++i) x = fmaf(sh.comb.w[h][i], gload(from + (int64_t)i * a.d.group * kHeadDim), x);
        const float l = sh.comb.l[h];
        const int64_t row = ((int64_t)b * a.d.n_kv_heads + g0) * a.d.group + sh.heads[h];
        gstore(a.out + row * kHeadDim + d, __builtin_bit_cast(uint16_t, (__bf16)(l == 0.0f ? 0.0f : x / l)));
    }
    __syncthreads();
}

template <int R, bool SETS, bool SCORES>
__global__ __launch_bounds__(kThreads, 2) void q4_attn_kernel(Q4AttnArgs a)
{
    __shared__ SharedQ4<R> sh;
    const int tid = threadIdx.x, B = a.d.batch, H = a.d.n_kv_heads;
    if (tid < kMaxKvHeads) {
        sh.rmask[tid] = a.rmask[tid];
        sh.rhead[tid] = a.rhead[tid];
        sh.ghead[tid] = a.ghead[tid];
    }
    int blocks = 0;
    if (tid < B) {
        const int L = clamp_tokens(gload(a.lengths + tid), a.d.max_len);
        sh.len[tid] = L;
        // (an empty segment is one block of tokens that do not count: its outputs are zero like any other's)
        blocks = a.n_rseg * max(1, (L + kQ4Block - 1) / kQ4Block) + a.n_gseg * max(1, (min(L, a.d.k) + kQ4Block - 1) / kQ4Block);
    }
    uint32_t total;
    const uint32_t upto = block_scan((uint32_t)blocks, sh.scan, total);
    if (tid < B) sh.pre[tid] = (int32_t)upto - blocks;
    if (tid == 0) sh.pre[B] = (int32_t)total;
    __syncthreads();
    const int T = uni((int)total);
    const int run = max(kWaves, (T + a.n_wg - 1) / a.n_wg);
    const int n_segs = a.n_rseg + a.n_gseg;
    int64_t x = (int64_t)blockIdx.x * run;
    const int64_t end = min(x + run, (int64_t)T);
    while (x < end) {
        const int b = uni(find_item(sh.pre, B, (int)x));
        const int L = uni(sh.len[b]);
        const int rb = max(1, (L + kQ4Block - 1) / kQ4Block);
        const int gb = max(1, (min(L, a.d.k) + kQ4Block - 1) / kQ4Block);
        const int rel = (int)x - uni(sh.pre[b]);
        const bool gather = SETS && rel >= a.n_rseg * rb;
        const int in = gather ? rel - a.n_rseg * rb : rel;
        const int per = gather ? gb : rb;
        const int si = in / per, j = in - si * per;
        const int nb = (int)min((int64_t)(per - j), end - x);
        const int g = uni((int)(gather ? sh.ghead[si] : sh.rhead[si]));
        uint32_t heads_mask = uni((uint32_t)sh.rmask[g]);
        if (gather) heads_mask = ~heads_mask & ((1u << a.d.group) - 1u);
        const int heads = __builtin_popcount(heads_mask);
        if (tid < kQ4MaxGroup && ((heads_mask >> tid) & 1u)) sh.heads[__builtin_popcount(heads_mask & ((1u << tid) - 1u))] = tid;
        __syncthreads();
        const int seg = b * n_segs + (gather ? a.n_rseg + si : si);
        const bool whole = nb == per;
        const int64_t slot = whole ? -1 : (int64_t)blockIdx.x + seg;
        Seq s;
        s.table = a.table + (int64_t)b * a.d.table_stride;
        s.set = SETS ? a.idx_in + ((int64_t)b * H + g) * a.d.k : nullptr;
        s.cache = a.cache;
        s.len = L;
        s.n = gather ? min(L, a.d.k) : L;
        s.head_tile = g << (a.d.page_shift - 4);
        if (SETS && gather) Piece<R, true, false>::run(a, s, b, g, heads, j, nb, slot, sh);
        else Piece<R, false, SCORES>::run(a, s, b, g, heads, j, nb, slot, sh);
        if (!whole) {
            if (tid == 0) {
                uint32_t *counter = a.seg_count + (((int64_t)b * H + g) * 2 + (gather ? 1 : 0)) * kLineWords;
                const uint32_t old = __hip_atomic_fetch_add((LYCHEE_GLOBAL uint32_t *)counter, (uint32_t)nb, __ATOMIC_RELAXED,
                                                            __HIP_MEMORY_SCOPE_AGENT);
                sh.last = old + (uint32_t)nb == (uint32_t)per;
                if (sh.last) gstore_through(counter, 0u);  // as every launch finds it
            }
            __syncthreads();
            if (sh.last) {
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
                const int64_t s0 = x - j;  // the segment's first block
                const int w0 = (int)(s0 / run), w1 = (int)((s0 + per - 1) / run);
                merge<R>(a, b, g, heads, (int64_t)w0 + seg, w1 - w0 + 1, sh);
            }
        }
        __syncthreads();
        x += nb;
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
    const int64_t rows = (int64_t)a.n_tokens * a.d.n_kv_heads;
    append_kernel<<<(uint32_t)((rows + kThreads / 16 - 1) / (kThreads / 16)), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_read(const ReadArgs &a, hipStream_t stream)
{
    const dim3 grid((uint32_t)((a.n_rows + kReadRows - 1) / kReadRows), (uint32_t)a.d.n_kv_heads, (uint32_t)a.d.batch);
    read_kernel<<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_q4_attn(const Q4AttnArgs &a, hipStream_t stream)
{
    return a.d.group <= 4 ? launch_r<1>(a, stream) : a.d.group <= 8 ? launch_r<2>(a, stream) : launch_r<4>(a, stream);
}

}  // namespace lychee
