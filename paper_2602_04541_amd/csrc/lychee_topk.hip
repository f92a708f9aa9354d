// Eq. 2 on rows of scores: the positions of the n = min(k, L) highest, ties to the lower position, in ascending order.
//
// A score's key is an unsigned integer that orders like it (NaN as -infinity, -0 as 0).  Three passes over the row count
// its keys' bits from the top, 11 + 11 + 10 at a time, and leave the n-th largest key and how many of the keys equal to it
// are taken; a fourth counts what every wavefront's stretch of the row contributes, and a fifth writes the positions.
#include "lychee_device.h"
#include "lychee_paged.h"

namespace lychee {
namespace {

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;

struct SharedTopk {
    uint32_t hist[2048];
    uint32_t wave[kSelWaves][2];
    uint32_t bin, left;
};

__device__ __forceinline__ uint32_t rank_key(float x)
{
    if (!(x == x)) return 0x007FFFFFu;  // a NaN: as -infinity
    return ordered_key(x + 0.0f);       // (-0 + 0 = 0)
}

__global__ __launch_bounds__(kSelThreads) void select_kernel(SelectArgs a)
{
    __shared__ SharedTopk sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int g = blockIdx.x % a.d.n_kv_heads, b = blockIdx.x / a.d.n_kv_heads;
    const int64_t row = (int64_t)b * a.d.n_kv_heads + g;
    int32_t *out = a.idx_out + row * a.d.k;
    const int k = a.d.k;
    if (!((a.selects >> g) & 1ull)) {
        const int32_t *in = a.idx_in + row * k;
        for (int i = tid; i < k; i += kSelThreads) gstore(out + i, gload(in + i));
        return;
    }
    int L = gload(a.lengths + b);
    L = L < 0 ? 0 : (L > a.d.max_len ? a.d.max_len : L);
    const int n = min(k, L);
    for (int i = n + tid; i < k; i += kSelThreads) gstore(out + i, -1);
    if (n == L) {
        for (int i = tid; i < n; i += kSelThreads) gstore(out + i, i);
        return;
    }
    const float *x = a.scores + row * a.score_stride;
    uint32_t prefix = 0, mask = 0, left = (uint32_t)n;  // keys with these top bits are undecided, `left` of them are taken
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int i = tid; i < 2048; i += kSelThreads) sh.hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < L; i += kSelThreads) {
            const uint32_t key = rank_key(gload(x + i));
            if ((key & mask) == prefix) atomicAdd(&sh.hist[(key >> shift) & ((1u << bits) - 1u)], 1u);
        }
        __syncthreads();
        // from the top: the bin in which the count reaches `left`; thread t has bins 2t and 2t+1, counted from the top
        const int last = (1 << bits) - 1;
        uint32_t c0 = 0, c1 = 0;
        if (2 * tid <= last) c0 = sh.hist[last - 2 * tid], c1 = sh.hist[last - 2 * tid - 1];
        const uint32_t in_wave = wave_scan(c0 + c1);
        if (lane == 63) sh.wave[wave][0] = in_wave;
        __syncthreads();
        uint32_t before = in_wave - (c0 + c1);
        for (int w = 0; w < wave; ++w) before += sh.wave[w][0];
        if (before < left && before + c0 >= left) {
            sh.bin = (uint32_t)(last - 2 * tid);
            sh.left = left - before;
        } else if (before + c0 < left && before + c0 + c1 >= left) {
            sh.bin = (uint32_t)(last - 2 * tid - 1);
            sh.left = left - before - c0;
        }
        __syncthreads();
        prefix |= sh.bin << shift;
        mask |= ((1u << bits) - 1u) << shift;
        left = sh.left;
        __syncthreads();
    }
    // prefix: the n-th largest key; `left` of the keys equal to it are taken, the lowest positions first
    const int per = (((L + kSelWaves - 1) / kSelWaves) + 63) & ~63;
    const int from = wave * per, to = min(L, from + per);
    uint32_t over = 0, same = 0;
    for (int i = from + lane; i < to; i += 64) {
        const uint32_t key = rank_key(gload(x + i));
        over += key > prefix;
        same += key == prefix;
    }
    over = wave_scan(over);
    same = wave_scan(same);
    if (lane == 63) {
        sh.wave[wave][0] = over;
        sh.wave[wave][1] = same;
    }
    __syncthreads();
    uint32_t at = 0, ties = 0;  // places taken before this wavefront's stretch, equal keys seen before it
    for (int w = 0; w < wave; ++w) {
        at += sh.wave[w][0];
        ties += sh.wave[w][1];
    }
    at += min(ties, left);
    for (int i0 = from; i0 < to; i0 += 64) {
        const int i = i0 + lane;
        const uint32_t key = i < to ? rank_key(gload(x + i)) : 0u;
        const unsigned long long eq = __ballot(i < to && key == prefix);
        const uint32_t mine = ties + (uint32_t)__builtin_popcountll(eq & ((1ull << lane) - 1ull));
        const bool take = i < to && (key > prefix || (key == prefix && mine < left));
        const unsigned long long all = __ballot(take);
        if (take) gstore(out + at + (uint32_t)__builtin_popcountll(all & ((1ull << lane) - 1ull)), i);
        at += (uint32_t)__builtin_popcountll(all);
        ties += (uint32_t)__builtin_popcountll(eq);
    }
}

}  // namespace

hipError_t launch_select(const SelectArgs &a, hipStream_t stream)
{
    select_kernel<<<(uint32_t)(a.d.batch * a.d.n_kv_heads), kSelThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace lychee
