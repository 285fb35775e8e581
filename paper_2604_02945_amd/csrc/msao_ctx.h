// msao_ctx.h -- the context behind the C ABI and what every entry point does
// with it: messages of failed calls, the device of the call, launches with
// profiling events. Shared by the host files; not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <initializer_list>
#include <string>
#include <utility>
#include <vector>

#include "../../include/msao.h"
#include "msao_internal.h"

namespace msao {

// Slots of pinned staging: so many uploads may be waiting on the GPU before
// the host waits for the oldest.
constexpr int kStageSlots = 4;

}  // namespace msao

struct msao_ctx {
    int device = 0;
    std::string err;
    // pinned staging slots, used in turn. The upload kernel's block b sets
    // stage_done[slot * kUploadMaxBlocks + b] to stage_ticket[slot] once it
    // has read the slot; until its stage_blocks[slot] blocks have, the slot
    // is not written again.
    void* stage[msao::kStageSlots] = {};
    size_t stage_cap[msao::kStageSlots] = {};
    uint32_t* stage_done = nullptr;   // pinned
    uint32_t stage_ticket[msao::kStageSlots] = {};
    int stage_blocks[msao::kStageSlots] = {};
    hipStream_t stage_stream[msao::kStageSlots] = {};
    int next_slot = 0;
    // slots in which the workgroups of a split row of logits meet. A call takes
    // one whose last user has set ent_done[slot] to ent_ticket[slot]
    msao::EntSlot* ent_slot[msao::kEntSlots] = {};
    uint32_t* ent_done = nullptr;     // pinned, behind stage_done
    uint32_t ent_ticket[msao::kEntSlots] = {};
    hipStream_t ent_stream[msao::kEntSlots] = {};
    int n_ent = 0, next_ent = 0;
    // profiling: an event pair around every launch, averaged per kernel on query
    bool profiling = false;
    std::vector<hipEvent_t> pool;                       // free events
    std::vector<std::pair<hipEvent_t, hipEvent_t>> rec[MSAO_NUM_KERNELS];
    std::vector<std::pair<hipEvent_t, hipEvent_t>> cache_rec[MSAO_NUM_CACHE_KERNELS];
    // tuning
    int row_item_bytes = 8192;
    int chain_frames = 0;       // frames per temporal work item; 0 = automatic
    int xcd_order = -1;         // scoring block order: -1 automatic, 0 dispatch order, 1 one range per XCD
    int clip_fuse = 1;          // the SimHash run scores and hashes its clips in one pass (k_clip)
    int pair_path = 1;          // clips with rows of at most 4 KiB are scored by k_pair
    int post_big_segment = msao::kPostBigSegment;  // selections this large take 1024-thread blocks
};

namespace msao {

inline thread_local std::string g_err;

inline constexpr size_t kWsAlign = 256;

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

inline int elt_size(int dtype) { return dtype == MSAO_F32 ? 4 : 2; }

inline msao_status fail(std::string* err, msao_status st, const std::string& msg)
{
    if (err) *err = msg;
    return st;
}

#define MSAO_TRY(x)                                                                                                   \
    do {                                                                                                              \
        msao_status st_ = (x);                                                                                        \
        if (st_ != MSAO_OK) return st_;                                                                               \
    } while (0)

inline msao_status hip_fail(msao_ctx* ctx, hipError_t e, const char* what)
{
    ctx->err = std::string(what) + ": " + hipGetErrorString(e);
    return MSAO_ERR_HIP;
}

struct DeviceGuard {
    int prev = -1;
    bool changed = false;
    explicit DeviceGuard(int dev)
    {
        if (hipGetDevice(&prev) == hipSuccess && prev != dev) changed = hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard()
    {
        if (changed) (void)hipSetDevice(prev);
    }
};

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p) % a == 0; }

// Output arrays of 4 or 8 bytes must be naturally aligned.
inline msao_status check_out_alignment(msao_ctx* ctx, std::initializer_list<std::pair<const void*, size_t>> ptrs)
{
    for (const auto& pr : ptrs)
        if (pr.first && !aligned(pr.first, pr.second))
            return fail(&ctx->err, MSAO_ERR_ALIGNMENT, "an output array is not naturally aligned");
    return MSAO_OK;
}

inline hipEvent_t pooled_event(msao_ctx* ctx)
{
    if (!ctx->pool.empty()) {
        hipEvent_t e = ctx->pool.back();
        ctx->pool.pop_back();
        return e;
    }
    hipEvent_t e = nullptr;
    return hipEventCreate(&e) == hipSuccess ? e : nullptr;
}

// Launch, with profiling events recorded at the kernel's start and end and kept in `rec`.
inline msao_status launched_in(msao_ctx* ctx, std::vector<std::pair<hipEvent_t, hipEvent_t>>& rec, hipStream_t stream,
                               int (*fn)(const void*, void*, void*, void*), const void* args)
{
    hipEvent_t e0 = nullptr, e1 = nullptr;
    if (ctx->profiling) {
        e0 = pooled_event(ctx);
        e1 = pooled_event(ctx);
        if (!e0 || !e1) return fail(&ctx->err, MSAO_ERR_HIP, "hipEventCreate failed");
    }
    const int rc = fn(args, stream, e0, e1);
    if (rc == kNoLaunch) {  // nothing to launch: the events were not recorded
        if (e0) ctx->pool.push_back(e0);
        if (e1) ctx->pool.push_back(e1);
        return MSAO_OK;
    }
    if (rc != 0) return hip_fail(ctx, (hipError_t)rc, "kernel launch");
    if (ctx->profiling) rec.push_back({e0, e1});
    return MSAO_OK;
}

inline msao_status launched(msao_ctx* ctx, int kernel, hipStream_t stream, int (*fn)(const void*, void*, void*, void*),
                            const void* args)
{
    return launched_in(ctx, ctx->rec[kernel], stream, fn, args);
}

// Mean milliseconds of the launches in `rec`, which is emptied.
inline msao_status mean_times(msao_ctx* ctx, std::vector<std::pair<hipEvent_t, hipEvent_t>>* rec, int n, float* ms)
{
    DeviceGuard guard(ctx->device);
    msao_status st = MSAO_OK;
    for (int k = 0; k < n; ++k) {
        double sum = 0.0;
        for (auto& pr : rec[k]) {
            float t = 0.0f;
            hipError_t e = hipEventSynchronize(pr.second);
            if (e == hipSuccess) e = hipEventElapsedTime(&t, pr.first, pr.second);
            if (e != hipSuccess && st == MSAO_OK) st = hip_fail(ctx, e, "msao_kernel_times");
            sum += t;
            ctx->pool.push_back(pr.first);
            ctx->pool.push_back(pr.second);
        }
        ms[k] = rec[k].empty() ? 0.0f : (float)(sum / (double)rec[k].size());
        rec[k].clear();
    }
    return st;
}

}  // namespace msao
