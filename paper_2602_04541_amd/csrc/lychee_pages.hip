// Bookkeeping of the paged cache on the GPU: finished requests' pages go back to the pool, a step's new tokens get
// pages and slots.
//
// Everything a request needs follows from prefix sums over the (at most 256) requests: with P tokens a page,
//     pages_b = ceil((L_b + n_b) / P) - ceil(L_b / P),   page_0_b = sum of pages before b,   start_b = sum of n before b,
// the j-th page a request takes is free_pages[count - 1 - page_0_b - j], and token i of the step belongs to the request
// with start_b <= i < start_b+1.  Every workgroup does the sums for itself (one thread a request: 1 KB of loads and a
// scan), so that none waits for another; what remains is spread over the workgroups by pages and by tokens.  Since
// lengths and free_count may be updated in place, they are written by the last workgroup to have read them (a value
// counts as read when it has been used: both go into LDS or into the scan ahead of the barrier in last_to_arrive).
#include "lychee_device.h"
#include "lychee_paged.h"

namespace lychee {
namespace {

static_assert(kThreads >= kMaxBatch, "one thread a request");

struct SharedPages {
    unsigned long long scan[kWaves + 1];
    int32_t page0[kMaxBatch + 1];   // pages of the requests before
    int32_t start[kMaxBatch + 1];   // tokens of the requests before
    int32_t len[kMaxBatch], held[kMaxBatch];
    int32_t count, bad, last;
};

__device__ __forceinline__ int clamp_tokens(int L, int most) { return L < 0 ? 0 : (L > most ? most : L); }

// Whether this workgroup is the last of the launch to come here; puts the counter back to zero.  Without a counter (the
// outputs are no inputs) it is the first one.
__device__ __forceinline__ bool last_to_arrive(uint32_t *arrived, int32_t *flag)
{
    __syncthreads();
    if (arrived == nullptr) return blockIdx.x == 0;
    if (threadIdx.x == 0) {
        const uint32_t n = __hip_atomic_fetch_add((LYCHEE_GLOBAL uint32_t *)arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *flag = n == gridDim.x - 1;
        if (*flag) gstore_through(arrived, 0u);
    }
    __syncthreads();
    return *flag != 0;
}

__global__ __launch_bounds__(kThreads) void release_kernel(ReleaseArgs a)
{
    __shared__ SharedPages sh;
    const int tid = threadIdx.x, B = a.d.batch, P = 1 << a.d.page_shift;
    int L = 0, back = 0;
    if (tid < B) {
        L = gload(a.lengths + tid);
        if (gload(a.done + tid)) {
            back = (clamp_tokens(L, a.d.max_len) + P - 1) >> a.d.page_shift;
            L = 0;
        }
    }
    if (tid == 0) sh.count = gload(a.free_count);
    unsigned long long total;
    const unsigned long long upto = block_scan64((unsigned long long)back, sh.scan, total);
    if (tid < B) sh.page0[tid] = (int32_t)upto - back;
    if (tid == 0) sh.page0[B] = (int32_t)total;
    const bool last = last_to_arrive(a.arrived, &sh.last);  // (and a barrier: page0 is whole)
    const int count = sh.count;
    const int base = count < 0 ? 0 : (count > a.d.n_pages ? a.d.n_pages : count);
    const int n = sh.page0[B];
    for (int i = blockIdx.x * kThreads + tid; i < n && base + i < a.d.n_pages; i += gridDim.x * kThreads) {
        const int b = find_item(sh.page0, B, i);
        gstore(a.free_pages + base + i, gload(a.table + (int64_t)b * a.d.table_stride + (i - sh.page0[b])));
    }
    if (last) {
        if (tid < B) gstore(a.lengths_out + tid, L);
        if (tid == 0) gstore(a.free_count_out, n == 0 ? count : min(base + n, a.d.n_pages));
    }
}

__global__ __launch_bounds__(kThreads) void plan_kernel(PlanArgs a)
{
    __shared__ SharedPages sh;
    const int tid = threadIdx.x, B = a.d.batch, shift = a.d.page_shift, P = 1 << shift;
    int L = 0, n = 0, held = 0, pages = 0;
    if (tid == 0) {
        sh.count = gload(a.free_count);
        sh.bad = sh.count < 0 || sh.count > a.d.n_pages;
    }
    __syncthreads();
    if (tid < B) {
        L = gload(a.lengths + tid);
        n = gload(a.new_tokens + tid);
        if (L < 0 || n < 0 || L > a.d.max_len || n > a.d.max_len - L) {
            sh.bad = 1;  // (every thread that writes writes the same)
            n = 0;
        } else {
            held = (L + P - 1) >> shift;
            pages = ((L + n + P - 1) >> shift) - held;
        }
    }
    // (256 requests of at most 2^24 tokens: 29 bits of pages, 33 of tokens)
    unsigned long long total;
    const unsigned long long mine = (unsigned long long)pages | ((unsigned long long)n << 30);
    const unsigned long long upto = block_scan64(mine, sh.scan, total);  // (barriers inside: sh.bad is whole after them)
    const int count = sh.count;
    const long long want_pages = (long long)(total & 0x3FFFFFFFull), want_tokens = (long long)(total >> 30);
    const int status = sh.bad ? -1 : want_tokens > a.n_slots ? -2 : want_pages > count ? (int)(want_pages - count) : 0;
    const bool ok = status == 0;
    if (tid < B) {
        const unsigned long long before = upto - mine;
        sh.page0[tid] = (int32_t)(before & 0x3FFFFFFFull);
        sh.start[tid] = (int32_t)(before >> 30);
        sh.len[tid] = L;
        sh.held[tid] = held;
    }
    if (tid == 0) {
        sh.page0[B] = (int32_t)want_pages;
        sh.start[B] = (int32_t)want_tokens;
    }
    const bool last = last_to_arrive(a.arrived, &sh.last);
    const int n_pages = ok ? (int)want_pages : 0, n_tokens = ok ? (int)want_tokens : 0;
    const int step = gridDim.x * kThreads;
    for (int i = blockIdx.x * kThreads + tid; i < n_pages; i += step) {
        const int b = find_item(sh.page0, B, i);
        gstore(a.table + (int64_t)b * a.d.table_stride + sh.held[b] + (i - sh.page0[b]), gload(a.free_pages + count - 1 - i));
    }
    // (n_slots may be 2^31 - 1, and a step goes past that)
    for (uint32_t at = blockIdx.x * kThreads + tid; at < (uint32_t)a.n_slots; at += step) {
        const int i = (int)at;
        int slot = -1;
        if (i < n_tokens) {
            const int b = find_item(sh.start, B, i);
            const int t = sh.len[b] + (i - sh.start[b]);
            const int e = t >> shift, fresh = e - sh.held[b];
            // (a page of this step is read where it was taken from: the table's entry may not be written yet)
            const int page = fresh >= 0 ? gload(a.free_pages + count - 1 - sh.page0[b] - fresh)
                                        : gload(a.table + (int64_t)b * a.d.table_stride + e);
            if ((uint32_t)page < (uint32_t)a.d.n_pages) slot = (page << shift) + (t & (P - 1));
        }
        gstore(a.slots + i, slot);
    }
    if (last) {
        if (tid < B) {
            gstore(a.lengths_out + tid, ok ? L + n : L);
            gstore(a.token_start + tid, ok ? sh.start[tid] : 0);
        }
        if (tid == 0) {
            gstore(a.token_start + B, n_tokens);
            gstore(a.free_count_out, count - n_pages);
            gstore(a.status, status);
        }
    }
}

// Workgroups for so many pages or slots: one a thread, since each is a chain of a search and two loads (four a thread, a
// step of 256 requests and 36K slots took 8.1 us instead of 5.2), but few where all of them count in on one word, 11 ns each
// (updated in place that step takes 8.7).
int grid_for(int64_t items, bool counted)
{
    const int64_t each = counted ? 4 * kThreads : kThreads, most = counted ? 64 : 512;
    const int64_t n = (items + each - 1) / each;
    return n < 1 ? 1 : n > most ? (int)most : (int)n;
}

}  // namespace

hipError_t launch_release(const ReleaseArgs &args, hipStream_t stream)
{
    ReleaseArgs a = args;
    const int64_t most = (int64_t)a.d.batch * (a.d.max_len >> a.d.page_shift);
    const bool in_place = a.lengths_out == a.lengths || a.free_count_out == a.free_count;
    const int grid = grid_for(most < a.d.n_pages ? most : a.d.n_pages, in_place);
    if (!in_place || grid == 1) a.arrived = nullptr;
    release_kernel<<<grid < 64 ? grid : 64, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_plan(const PlanArgs &args, hipStream_t stream)
{
    PlanArgs a = args;
    const bool in_place = a.lengths_out == a.lengths || a.free_count_out == a.free_count;
    const int grid = grid_for(a.n_slots, in_place);
    if (!in_place || grid == 1) a.arrived = nullptr;
    plan_kernel<<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace lychee
