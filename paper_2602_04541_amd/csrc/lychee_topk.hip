// Eq. 2 on rows of scores: the positions of the n = min(k, L) highest, ties to the lower position, in ascending order.
//
// A score's key is an unsigned integer that orders like it (NaN as -infinity, -0 as 0).  One workgroup a row; thread t has
// positions t, t + 1024, ..
//   1  The row is cut into groups, each thread's consecutive positions, about 2n of them where the row is long enough
//      (topk_group).
//      The n-th largest of the groups' largest keys is a bound that n keys at least reach, whatever the scores are, and for
//      scores without order about 1.4 n (G groups of which n reach it hold -G ln(1 - n/G) keys above).  So only the groups'
//      largest are counted, an eighth of an octave a bin, and the rest of the row meets one comparison a key.
//   2  Scores from the bound on are the candidates: a list of them in LDS, a share of it for every wavefront, and a count of
//      their keys in 4096 even bins.  The bin in which the count from the top reaches n holds the n-th largest; again within
//      that bin while it holds more than are ranked at once.
//   3  Candidates above the bin go into a bitmap of positions.  The bin's own few are ranked against one another; or, if all
//      of them are taken, treated like those above; or, if they are one key, they have a bitmap of their own, whose first so
//      many count.
//   4  A prefix sum over the bitmap's words gives every word its place in the set.
// Rows of up to 8 positions a thread stay in registers between 1 and 2; longer ones are read again, from the L2 (32 positions a
// thread in registers are 0.6 us slower for a row of 32K).  Where the candidates are more than the list holds (many equal
// scores, sets of more than 8000) or the row is longer than the bitmap, 2 and 3 go over the row itself instead, a window of the
// bitmap at a time (select_scan): 10000 of a row of 32768 take 27 us, 16384 of 131072 68, 4096 of 262144 105.
//
// Bound by one CU's work on its row: a row of 32768 scores takes 14.1 us for 2048 of them and 11.5 for 256 (32 without
// step 1's bound), 64 rows of up to 98304 25.3 for 4096, of which the passes over the row have half, and the chains of barriers,
// prefix sums and LDS atomics the rest; the bytes are 2 us of it.  One way to share a row was tried: up to 8 workgroups list
// candidates, the last one selects from the lists; 17.9 and 45 us, since that one's chain is as long as a row's of its own.
#include "lychee_device.h"
#include "lychee_paged.h"

namespace lychee {
namespace {

constexpr int kSelThreads = kTopkThreads;
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kTopBins = 4096;
constexpr int kBinsEach = kTopBins / kSelThreads;  // bins a thread adds up
constexpr int kTopList = 512;                      // keys that are ranked against one another
constexpr int kWindow = 1 << 17;                   // positions the bitmaps hold
constexpr int kWindowWords = kWindow / 64;
constexpr int kCandEach = 768;                     // candidates a wavefront lists

struct SharedTopk {
    uint32_t hist[kTopBins];
    unsigned long long above[kWindowWords], ties[kWindowWords];
    unsigned long long list[kTopList];  // key, ~position
    uint32_t cand[kSelWaves][kCandEach];  // positions
    uint32_t wave[kSelWaves], top[kSelWaves];
    uint32_t bin, left, count, n_list, full;
};

__device__ __forceinline__ uint32_t rank_key(float x)
{
    if (!(x == x)) return 0x007FFFFFu;  // a NaN: as -infinity
    return ordered_key(x + 0.0f);       // (-0 + 0 = 0)
}

// Inclusive prefix sum over the workgroup; `total` = sum of all.
__device__ __forceinline__ uint32_t scan_1024(uint32_t v, SharedTopk &sh, uint32_t &total)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t x = wave_scan(v);
    __syncthreads();
    if (lane == 63) sh.wave[wave] = x;
    __syncthreads();
    const uint32_t t = sh.wave[lane & (kSelWaves - 1)];
    const uint32_t upto = wave_scan(lane < kSelWaves ? t : 0u);
    total = (uint32_t)__builtin_amdgcn_readlane((int)upto, kSelWaves - 1);
    return x + (wave > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)upto, uni(wave) - 1) : 0u);
}

// The bin in which the count from the top reaches `want` (>= 1, no more than all): sh.bin, what is left to take in it
// (sh.left) and what it holds (sh.count).  Clears the bins.
__device__ __forceinline__ void find_bin(uint32_t want, SharedTopk &sh)
{
    const int tid = threadIdx.x;
    __syncthreads();
    const int top = kTopBins - kBinsEach * (tid + 1);  // thread 0 has the last bins
    uint4 c = *reinterpret_cast<uint4 *>(&sh.hist[top]);
    *reinterpret_cast<uint4 *>(&sh.hist[top]) = make_uint4(0, 0, 0, 0);
    uint32_t total;
    const uint32_t mine = c.x + c.y + c.z + c.w;
    uint32_t before = scan_1024(mine, sh, total) - mine;
    if (before < want && before + mine >= want) {
        const uint32_t in[4] = {c.w, c.z, c.y, c.x};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (before < want && before + in[i] >= want) {
                sh.bin = (uint32_t)(top + 3 - i);
                sh.left = want - before;
                sh.count = in[i];
            }
            before += in[i];
        }
    }
    __syncthreads();
}

// A row's scores: position i * 1024 + t of the row is number i of thread t.  A NaN is -infinity; behind the row's end there are
// NaN, which no comparison takes.  Scores are compared as they are, an instruction each; keys are for those that count.
// (A comparison: fmaxf is free to give a signaling NaN back.)
__device__ __forceinline__ float number(float x) { return x == x ? x : -__builtin_inff(); }
__device__ __forceinline__ float score_at(float x, int pos, int i, int L)
{
    x = number(x);
    if ((i + 1) * kSelThreads > L) x = pos < L ? x : __builtin_nanf("");  // (uniform: a thread's last)
    return x;
}
template <int E>
struct Scores {  // in registers
    float x[E];
    int n;  // of every thread
    __device__ __forceinline__ Scores(const float *p, int L, int tid) : n((L + kSelThreads - 1) / kSelThreads)
    {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (i % 8 == 0 && i >= n) break;  // (uniform)
            x[i] = gload(p + min(i * kSelThreads + tid, L - 1));
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (i % 8 == 0 && i >= n) break;
            x[i] = score_at(x[i], i * kSelThreads + tid, i, L);
        }
        for (int i = 0; i < E; ++i)
            if (i >= ((n + 7) & ~7)) x[i] = __builtin_nanf("");
    }
    // f(i, score) for the numbers [from, to) of every thread, and some NaN; all of the workgroup's threads together
    template <typename F>
    __device__ __forceinline__ void for_each(int, int, F f) const
    {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (i % 8 == 0 && i >= n) break;
            f(i, x[i]);
        }
    }
    // f(i0, x): numbers i0 .. of every thread, an array of them (behind the thread's last: NaN)
    template <typename F>
    __device__ __forceinline__ void in_batches(F f) const { f(0, x); }
};
template <>
struct Scores<0> {  // read again
    const float *p;
    int L, tid, n;
    __device__ __forceinline__ Scores(const float *p_, int L_, int tid_) : p(p_), L(L_), tid(tid_), n((L_ + kSelThreads - 1) / kSelThreads) {}
    template <typename F>
    __device__ __forceinline__ void for_each(int from, int to, F f) const
    {
        constexpr int kU = 24;  // loads in flight: the L2 is 0.7 us away, and a workgroup alone has to draw on it
        const int whole = L / kSelThreads;  // numbers that every thread has
        int i0 = from;
        for (; i0 + kU <= min(to, whole); i0 += kU) {
            const float *q = uni(p + (int64_t)i0 * kSelThreads);
            float v[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) v[u] = gload(q + (uint32_t)(u * kSelThreads + tid));
#pragma unroll
            for (int u = 0; u < kU; ++u) f(i0 + u, number(v[u]));
        }
        for (; i0 < to; i0 += 8) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = gload(p + min((i0 + u) * kSelThreads + tid, L - 1));
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i0 + u < to) f(i0 + u, score_at(v[u], (i0 + u) * kSelThreads + tid, i0 + u, L));
        }
    }
    template <typename F>
    __device__ __forceinline__ void in_batches(F f) const
    {
        constexpr int kU = 32;
        for (int i0 = 0; i0 < n; i0 += kU) {
            float v[kU];
            if ((i0 + kU) * kSelThreads <= L) {
                const float *q = uni(p + (int64_t)i0 * kSelThreads);
#pragma unroll
                for (int u = 0; u < kU; ++u) v[u] = gload(q + (uint32_t)(u * kSelThreads + tid));
            } else {
#pragma unroll
                for (int u = 0; u < kU; ++u) v[u] = gload(p + min((i0 + u) * kSelThreads + tid, L - 1));
#pragma unroll
                for (int u = 0; u < kU; ++u) v[u] = (i0 + u) * kSelThreads + tid < L ? v[u] : __builtin_nanf("");
            }
            f(i0, v);
        }
    }
};

// The score of a key between those of the infinities.
__device__ __forceinline__ float score_of(uint32_t key)
{
    return __builtin_bit_cast(float, (key & 0x80000000u) ? key & 0x7FFFFFFFu : ~key);
}
constexpr uint32_t kLeastKey = 0x007FFFFFu;  // of -infinity
// The score that bounds the keys up to this one: the key behind the negative numbers' is no score's, and as a number it would
// be the -0 that compares equal to the +0 above it.
__device__ __forceinline__ float score_up_to(uint32_t key) { return score_of(key == 0x7FFFFFFFu ? key - 1u : key); }

// Ranks the keys in sh.list (c of them) against one another and marks the positions of the `left` largest.
__device__ __forceinline__ void rank_list(uint32_t c, uint32_t left, SharedTopk &sh)
{
    for (uint32_t e = threadIdx.x; e < c; e += kSelThreads) {
        const unsigned long long mine = sh.list[e];
        uint32_t before = 0;
        for (uint32_t j = 0; j < c; ++j) before += sh.list[j] > mine;
        const uint32_t pos = ~(uint32_t)mine;
        if (before < left) atomicOr(&sh.above[pos >> 6], 1ull << (pos & 63u));
    }
    __syncthreads();
}

// Writes the positions marked in a window's first `words` words, which begins at position w0, behind the `at` places taken;
// tied: of the positions marked in sh.ties the lowest ones too, `left` in all, `ties` of them in windows before.
__device__ __forceinline__ void place(int32_t *out, int w0, int words, bool tied, uint32_t left, uint32_t &at, uint32_t &ties, SharedTopk &sh)
{
    const int tid = threadIdx.x;
    unsigned long long b[2];  // thread t has words 2t and 2t + 1 of the window's 2048
    uint32_t total = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) b[u] = 2 * tid + u < words ? sh.above[2 * tid + u] : 0ull;
    if (tied) {
        unsigned long long t[2];
        uint32_t c[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            t[u] = 2 * tid + u < words ? sh.ties[2 * tid + u] : 0ull;
            c[u] = (uint32_t)__builtin_popcountll(t[u]);
        }
        uint32_t seen = scan_1024(c[0] + c[1], sh, total) - c[0] - c[1] + ties;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (seen + c[u] <= left) {
                b[u] |= t[u];
            } else {  // the lowest ones that are still to take
                for (uint32_t i = seen; i < left; ++i) {
                    b[u] |= t[u] & (0ull - t[u]);
                    t[u] &= t[u] - 1;
                }
            }
            seen += c[u];
        }
        ties += total;
    }
    const uint32_t mine = (uint32_t)__builtin_popcountll(b[0]) + (uint32_t)__builtin_popcountll(b[1]);
    uint32_t place = scan_1024(mine, sh, total) - mine + at;
    at += total;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int p0 = w0 + (2 * tid + u) * 64;
        for (unsigned long long m = b[u]; m != 0; m &= m - 1) gstore(out + place++, p0 + (int)__builtin_ctzll(m));
    }
    __syncthreads();
}

// Steps 2 to 4 over the row itself; lo, hi: keys that the n-th largest and the largest lie between.
__device__ __forceinline__ void select_scan(const float *x, int L, int n, uint32_t lo, uint32_t hi, int32_t *out, SharedTopk &sh)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const Scores<0> row(x, L, tid);
    uint32_t left = (uint32_t)n, count;
    int shift;
    for (;;) {
        const uint32_t span = hi - lo;
        shift = span < (uint32_t)kTopBins ? 0 : 20 - __builtin_clz(span);
        const float from = score_of(lo), to = score_up_to(hi);
        __syncthreads();
        // (from +0 on a score orders like its bits, -0 aside)
        if (lo >= 0x80000000u) {
            row.for_each(0, row.n, [&](int, float v) {
                if (v >= from && v <= to) atomicAdd(&sh.hist[(__builtin_bit_cast(uint32_t, v + 0.0f) - (lo & 0x7FFFFFFFu)) >> shift], 1u);
            });
        } else {
            row.for_each(0, row.n, [&](int, float v) {
                if (v >= from && v <= to) atomicAdd(&sh.hist[(rank_key(v) - lo) >> shift], 1u);
            });
        }
        find_bin(left, sh);
        lo += sh.bin << shift;
        hi = min(hi, lo + ((1u << shift) - 1u));
        left = sh.left;
        count = sh.count;
        if (shift == 0 || count == left || (count <= (uint32_t)kTopList && L <= kWindow)) break;
    }
    const bool whole = count == left, ranked = !whole && shift != 0;
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    // 3 and 4, a window of positions at a time
    uint32_t at = 0, ties = 0;  // places and ties of the windows before
    // (what lies above: from lo on, if the bin is taken whole, else from the key behind hi on)
    const float bin_lo = score_of(lo), bin_hi = score_up_to(hi);
    for (int w0 = 0; w0 < L; w0 += kWindow) {
        const int from = w0 / kSelThreads, to = min(row.n, from + kWindow / kSelThreads);
        uint32_t al = 0, ah = 0, tl = 0, th = 0;  // 64 numbers' words, one a lane
        auto put = [&](int i_last) {
            const int i = (i_last & ~63) + lane;
            if (i <= i_last && i < to) {
                sh.above[(i - from) * kSelWaves + wave] = ((unsigned long long)ah << 32) | al;
                sh.ties[(i - from) * kSelWaves + wave] = ((unsigned long long)th << 32) | tl;
            }
        };
        row.for_each(from, to, [&](int i, float v) {
            const unsigned long long in = __ballot(v >= bin_lo), over = __ballot(v > bin_hi);
            const unsigned long long a = whole ? in : over, t = in & ~a;
            const bool mine = lane == (i & 63);
            al = mine ? (uint32_t)a : al;
            ah = mine ? (uint32_t)(a >> 32) : ah;
            if (t != 0) {  // (few)
                tl = mine ? (uint32_t)t : tl;
                th = mine ? (uint32_t)(t >> 32) : th;
                if (ranked && ((t >> lane) & 1ull))
                    sh.list[atomicAdd(&sh.n_list, 1u)] = ((unsigned long long)rank_key(v) << 32) | (uint32_t)~(i * kSelThreads + tid);
            }
            if ((i & 63) == 63) {
                put(i);
                tl = th = 0;
            }
        });
        if ((to & 63) != 0) put(to - 1);
        __syncthreads();
        if (ranked) rank_list(sh.n_list, left, sh);
        place(out, w0, (to - from) * kSelWaves, !whole && !ranked, left, at, ties, sh);
    }
}

template <int E>
__device__ __forceinline__ void select_row(const float *x, int L, int n, int32_t *out, SharedTopk &sh)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const Scores<E> row(x, L, tid);
    // 1: groups of `each` scores
    const int each = topk_group(n, L);
    {
        float m = __builtin_nanf(""), most = m;
        int left = each;
        row.for_each(0, row.n, [&](int i, float v) {
            m = fmaxf(m, v);
            if (--left == 0 || i == row.n - 1) {
                if (m == m) atomicAdd(&sh.hist[rank_key(m) >> 20], 1u);
                most = fmaxf(most, m);
                m = __builtin_nanf("");
                left = each;
            }
        });
        const uint32_t top = wave_max(most == most ? rank_key(most) : 0u);
        if (lane == 0) sh.top[wave] = top;
    }
    __syncthreads();
    uint32_t hi = wave_max(sh.top[lane & (kSelWaves - 1)]);
    find_bin((uint32_t)n, sh);  // (at least n groups have been counted: topk_group)
    uint32_t lo = max(kLeastKey, sh.bin << 20);
    // 2: the candidates.  A thread marks its own in a word, 32 positions at a time, and the wavefront's go into its list at a
    // prefix sum of their numbers; then they are dealt to its lanes.  (With a branch for every 64 scores that hold a candidate,
    // and nearly all do, a row of 98K took 17 us here.)  A bound of -infinity leaves out nothing.
    const bool listed = L <= kWindow && lo > kLeastKey;
    int used = 0;  // of the wavefront's list
    if (tid == 0) sh.full = 0;
    if (listed) {
        const int words = (L + 63) / 64;
        for (int i = tid; i < words; i += kSelThreads) sh.above[i] = sh.ties[i] = 0;
    }
    __syncthreads();
    uint32_t left = (uint32_t)n, count;
    int shift = hi - lo < (uint32_t)kTopBins ? 0 : 20 - __builtin_clz(hi - lo);
    constexpr int kHeld = kCandEach / 64;  // candidates of a lane
    uint32_t key[kHeld], pos[kHeld];
    if (listed) {
        const float bound = score_of(lo);
        row.in_batches([&](int i0, const auto &v) {
            constexpr int kU = sizeof v / sizeof v[0];
            uint32_t mask = 0;
#pragma unroll
            for (int u = 0; u < kU; ++u) mask |= v[u] >= bound ? 1u << u : 0u;
            const int c = __builtin_popcount(mask);
            const int upto = (int)wave_scan((uint32_t)c);
            int at = used + upto - c;
            used += __builtin_amdgcn_readlane(upto, 63);
            for (; mask != 0; mask &= mask - 1, ++at)
                if (at < kCandEach) sh.cand[wave][at] = (uint32_t)((i0 + __builtin_ctz(mask)) * kSelThreads + tid);
        });
        if (used > kCandEach && lane == 0) sh.full = 1;
        used = min(used, kCandEach);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        float v[kHeld];
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            if (u * 64 >= used) break;  // (uniform)
            pos[u] = sh.cand[wave][min(u * 64 + lane, used - 1)];
            v[u] = gload(x + pos[u]);
        }
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            if (u * 64 >= used) break;
            key[u] = u * 64 + lane < used ? rank_key(v[u]) : 0u;
            if (key[u] != 0) atomicAdd(&sh.hist[(key[u] - lo) >> shift], 1u);
        }
    }
    __syncthreads();
    if (!listed || sh.full) {
        for (int i = tid; i < kTopBins; i += kSelThreads) sh.hist[i] = 0;
        select_scan(x, L, n, lo, hi, out, sh);
        return;
    }
    for (;;) {
        find_bin(left, sh);
        lo += sh.bin << shift;
        hi = min(hi, lo + ((1u << shift) - 1u));
        left = sh.left;
        count = sh.count;
        if (shift == 0 || count == left || count <= (uint32_t)kTopList) break;
        shift = hi - lo < (uint32_t)kTopBins ? 0 : 20 - __builtin_clz(hi - lo);
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            if (u * 64 >= used) break;
            if (key[u] - lo <= hi - lo) atomicAdd(&sh.hist[(key[u] - lo) >> shift], 1u);
        }
    }
    // 3
    const bool whole = count == left, ranked = !whole && shift != 0;
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
        if (u * 64 >= used) break;
        if (key[u] < lo) continue;
        if (key[u] > hi || whole) atomicOr(&sh.above[pos[u] >> 6], 1ull << (pos[u] & 63u));
        else if (ranked) sh.list[atomicAdd(&sh.n_list, 1u)] = ((unsigned long long)key[u] << 32) | ~pos[u];
        else atomicOr(&sh.ties[pos[u] >> 6], 1ull << (pos[u] & 63u));
    }
    __syncthreads();
    if (ranked) rank_list(sh.n_list, left, sh);
    uint32_t at = 0, ties = 0;
    place(out, 0, (L + 63) / 64, !whole && !ranked, left, at, ties, sh);
}

__global__ __launch_bounds__(kSelThreads) void select_kernel(SelectArgs a)
{
    __shared__ __align__(16) SharedTopk sh;
    const int tid = threadIdx.x;
    const int g = blockIdx.x % a.d.n_kv_heads, b = blockIdx.x / a.d.n_kv_heads;
    const int64_t r = (int64_t)b * a.d.n_kv_heads + g;
    int32_t *out = a.idx_out + r * a.d.k;
    const int k = a.d.k;  // (up to 2^31 - 1: loops up to it step past an int's range)
    if (!((a.selects >> g) & 1ull)) {
        const int32_t *in = a.idx_in + r * k;
        for (uint32_t i = tid; i < (uint32_t)k; i += kSelThreads) gstore(out + i, gload(in + i));
        return;
    }
    int L = uni(gload(a.lengths + b));
    L = L < 0 ? 0 : (L > a.d.max_len ? a.d.max_len : L);
    const int n = min(k, L);
    for (uint32_t i = n + tid; i < (uint32_t)k; i += kSelThreads) gstore(out + i, -1);
    if (n == L) {
        for (int i = tid; i < n; i += kSelThreads) gstore(out + i, i);
        return;
    }
    for (int i = tid; i < kTopBins; i += kSelThreads) sh.hist[i] = 0;
    __syncthreads();
    const float *x = a.scores + r * a.score_stride;
    if (L <= 8 * kSelThreads) select_row<8>(x, L, n, out, sh);
    else select_row<0>(x, L, n, out, sh);
}

}  // namespace

hipError_t launch_select(const SelectArgs &a, hipStream_t stream)
{
    select_kernel<<<(uint32_t)(a.d.batch * a.d.n_kv_heads), kSelThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace lychee
