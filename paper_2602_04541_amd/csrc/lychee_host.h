// What the host sides of the paged cache and of attention over prompts share.
#pragma once

#include "lychee_context.h"
#include "lychee_paged.h"

namespace lychee {
namespace {

PagedDims dims_of(const lychee_paged &p)
{
    PagedDims d;
    d.batch = p.batch;
    d.n_kv_heads = p.n_kv_heads;
    d.group = p.n_q_heads / p.n_kv_heads;
    d.n_pages = p.n_pages;
    d.page_shift = 0;
    while ((1 << d.page_shift) < p.page_size) ++d.page_shift;
    d.max_len = p.max_pages * p.page_size;
    d.table_stride = p.table_stride;
    d.page_tiles = p.page_tiles;
    d.k = p.k;
    return d;
}

// The context's device while a call launches, then the caller's again.
struct OnDevice {
    int before = -1;
    bool ok = false;
    explicit OnDevice(const lychee_ctx *ctx)
    {
        ok = hipGetDevice(&before) == hipSuccess && (before == ctx->device || hipSetDevice(ctx->device) == hipSuccess);
        if (before == ctx->device) before = -1;
    }
    ~OnDevice()
    {
        if (before >= 0) (void)hipSetDevice(before);
    }
    OnDevice(const OnDevice &) = delete;
    OnDevice &operator=(const OnDevice &) = delete;
};

int done(hipError_t e) { return e == hipSuccess ? LYCHEE_OK : LYCHEE_EHIP; }

}  // namespace
}  // namespace lychee
