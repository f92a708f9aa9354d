// The context behind the C ABI, shared by the files of its host side, and what lies where in its device memory.
#pragma once

#include "../../include/lychee.h"
#include "lychee_internal.h"

#include <stddef.h>
#include <stdint.h>

#include <vector>

struct lychee_ctx {
    int device = 0;
    int n_cu = 256;
    int32_t wg_per_cu = 2;
    int32_t n_wg = 0;          // 0 = n_cu * wg_per_cu
    int32_t step_mode = LYCHEE_STEP_PHASED;
    int32_t g_block_rows = 0;  // 0: by the context's length, see fill_common
    int32_t tail_permille = 250;
    int32_t select_margin = 60;  // tenths of a standard deviation, see LYCHEE_OPT_SELECT_MARGIN
    int32_t select_lead = 3000;  // blocks of 64 rows streamed while a select runs, see LYCHEE_OPT_SELECT_LEAD
    int32_t wait_polls = lychee::kWaitPolls;
    uint32_t launch_seq = 0;   // pooled launches so far: picks the chunk counter
    std::vector<int32_t> used_slots;  // counters of pooled launches that no later launch has reset yet
    bool timing = false;
    struct Rec {
        int cls;
        hipEvent_t start, stop;
    };
    std::vector<Rec> recs;         // events recorded since the last read
    std::vector<hipEvent_t> pool;  // events free for reuse
    // Descriptor tables: built on the host, staged in pinned memory, copied to the arena
    // with an asynchronous copy on the caller's stream, and cached by content so that a
    // serving loop that passes the same buffers every step uploads nothing.
    void *static_scratch = nullptr;  // this device's address of the file-scope scratch array
    // What the workgroups of a layer launch hand to one another (zeroed once, then kept clean by
    // the launches themselves): the launch generation, the threshold and set flags, the
    // segments' arrival counters, and three banks of candidate counters (banks 0 and 1 alternate
    // between the layer calls that leave their select pending; calls that do not, and the layers of a
    // layer-after-layer step, use bank 2 and whichever of the others no pending select owns).
    char *sync_dev = nullptr;
    char *arena_dev = nullptr;
    char *arena_host = nullptr;  // pinned, same layout as the device arena
    size_t arena_used = 0;
    bool arena_captured = false;  // some table was uploaded or used while a stream was being captured
    struct Cached {
        uint64_t hash;
        size_t offset, bytes;
    };
    std::vector<Cached> cache;
    std::vector<lychee::LayerDesc> descs;  // a call's layer descriptors (capacity for the most layers a step takes)
    // A layer call whose select has been left for the next call (lychee_decode_attn_deferred).
    struct Pending {
        bool active = false;
        lychee::LayerDesc desc;              // the layer, its queries redirected to the workspace's copy
        lychee_shape shape;
        const int32_t *lengths = nullptr;
        void *workspace = nullptr;
        int slot = 0;                // which of the workspace's two layer slots holds its scratch
        int bank = 0;                // which bank of candidate counters it collected into
    } pending;
};

namespace lychee {

// Layout of lychee_ctx::sync_dev
constexpr size_t kSyncGen = 0, kSyncApart = 128, kSyncExit = 256;  // uint32 [1 + kExitGroups], lines of their own
constexpr size_t kSyncRows = (size_t)kMaxBatch * kMaxKvHeads;  // (sequence, KV head) pairs a shape can have
constexpr size_t kSyncThr = 8192;                               // uint64 [kSyncRows][kLineWords / 2]
constexpr size_t kSyncPages = kSyncExit + 4 * kLineWords * (1 + kExitGroups);  // uint32: workgroups that have read a plan's inputs
static_assert(kSyncPages + 4 * kLineWords <= kSyncThr, "");
constexpr size_t kSyncSet = kSyncThr + kSyncRows * kLineWords * 4;  // uint32 [kSetFlagWords]
constexpr size_t kSyncSeg = kSyncSet + kSetFlagWords * 4;  // uint32 [kSyncRows][2][kLineWords]
constexpr size_t kSyncCount = kSyncSeg + kSyncRows * 2 * kLineWords * 4;  // int32 [3][kSyncRows][kLineWords]
constexpr size_t kSyncArrived = kSyncCount + 3 * kSyncRows * kLineWords * 4;  // uint32 [kSyncRows][kLineWords]
constexpr size_t kSyncBytes = kSyncArrived + kSyncRows * kLineWords * 4;

inline int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

}  // namespace lychee
