// msao_sample_host.cpp -- host side of the entry points that draw tokens and verify
// drafts: checks of arguments before anything is enqueued, workspaces.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <string>

#include "../../include/msao.h"
#include "msao_ctx.h"
#include "msao_internal.h"
#include "msao_sample.h"

using namespace msao;

namespace {

constexpr int64_t kMaxRows = (1 << 24) - 1;
constexpr int64_t kMaxRowStride = (int64_t)1 << 31;

// A call that the C ABI must not leave by an exception.
template <typename F>
msao_status guarded(F f)
{
    try {
        return f();
    } catch (...) {
        return MSAO_ERR_HIP;
    }
}

msao_status bad(std::string* err, const char* what) { return fail(err, MSAO_ERR_INVALID_ARG, what); }

msao_status check_vocab(int64_t vocab, int dtype, std::string* err)
{
    if (dtype != MSAO_F32 && dtype != MSAO_BF16) return bad(err, "unknown dtype");
    if (vocab < 1) return bad(err, "vocab < 1");
    if (vocab > kMaxVocab) return fail(err, MSAO_ERR_UNSUPPORTED, "a vocabulary of more than 2^20 tokens");
    return MSAO_OK;
}

msao_status check_logits(const void* p, int64_t rows, int64_t vocab, int64_t stride, int dtype, const char* name, std::string* err)
{
    if (stride < vocab || stride > kMaxRowStride) return fail(err, MSAO_ERR_INVALID_ARG, std::string("the row stride of ") + name + " is out of range");
    if (rows > 0 && !p) return fail(err, MSAO_ERR_INVALID_ARG, std::string(name) + " is NULL");
    if (!aligned(p, 16) || stride * elt_size(dtype) % 16 != 0)
        return fail(err, MSAO_ERR_ALIGNMENT, std::string(name) + " or its row pitch is not a multiple of 16 bytes");
    return MSAO_OK;
}

msao_status check_words(std::initializer_list<const void*> ptrs, std::string* err)
{
    for (const void* p : ptrs)
        if (!aligned(p, 4)) return fail(err, MSAO_ERR_ALIGNMENT, "an array is not 4-byte aligned");
    return MSAO_OK;
}

msao_status check_set(const msao_sampling* set, SamplingDev& d, std::string* err)
{
    d = SamplingDev{nullptr, nullptr, nullptr, nullptr};
    if (set) d = SamplingDev{set->temperature, set->top_k, set->top_p, set->min_p};
    return check_words({d.temperature, d.top_k, d.top_p, d.min_p}, err);
}

msao_status check_workspace(void* ws, size_t given, size_t needed, std::string* err)
{
    if (needed == 0) return MSAO_OK;
    if (!ws) return fail(err, MSAO_ERR_WORKSPACE, "workspace is NULL");
    if (!aligned(ws, kWsAlign)) return fail(err, MSAO_ERR_WORKSPACE, "workspace is not 256-byte aligned");
    if (given < needed)
        return fail(err, MSAO_ERR_WORKSPACE, "workspace too small: " + std::to_string(given) + " bytes given, " + std::to_string(needed) + " needed");
    return MSAO_OK;
}

msao_status check_rows_count(int64_t rows, std::string* err)
{
    if (rows < 0) return bad(err, "rows is negative");
    if (rows > kMaxRows) return fail(err, MSAO_ERR_UNSUPPORTED, "2^24 rows or more");
    return MSAO_OK;
}

// Offsets of the arrays that the rows' first reading leaves.
struct ScanPlan {
    ScanDev scan;
    size_t most, sum, of, number, total;
};
ScanPlan scan_plan(int64_t work, int64_t rows, int64_t vocab, int dtype)
{
    ScanPlan pl;
    std::memset(&pl, 0, sizeof pl);
    scan_shape(pl.scan, work, vocab, dtype);
    pl.sum = 0;
    pl.most = pl.sum + align_up((size_t)rows * (size_t)pl.scan.segments * 8, kWsAlign);
    pl.of = pl.most + align_up((size_t)rows * (size_t)pl.scan.shares * 4, kWsAlign);
    pl.number = pl.of + align_up((size_t)rows * (size_t)pl.scan.segments * 4, kWsAlign);
    pl.total = pl.number + align_up((size_t)rows * (size_t)pl.scan.segments * 4, kWsAlign);
    return pl;
}
ScanDev scan_at(const ScanPlan& pl, uint8_t* ws)
{
    ScanDev d = pl.scan;
    if (d.parts > 0) {
        d.sum = (double*)(ws + pl.sum);
        d.most = (float*)(ws + pl.most);
        d.of = (float*)(ws + pl.of);
        d.number = (int32_t*)(ws + pl.number);
    }
    return d;
}

// Offsets of a verification's workspace arrays.
struct VerifyPlan {
    ScanPlan scan;
    size_t token, logprob, yes, known, total;
    int32_t max_new;
};
msao_status verify_plan(const msao_chunk* ch, int32_t n_seqs, int64_t vocab, int dtype, VerifyPlan& pl, std::string* err)
{
    if (!ch) return bad(err, "chunk is NULL");
    if (ch->n_rows < 0 || ch->max_new < 0 || n_seqs < 0) return bad(err, "a count is negative");
    MSAO_TRY(check_vocab(vocab, dtype, err));
    pl.max_new = std::min(ch->max_new, ch->n_rows);
    if ((int64_t)n_seqs * std::max(pl.max_new, 1) > kMaxRows) return fail(err, MSAO_ERR_UNSUPPORTED, "2^24 rows or more");
    const size_t rows = align_up((size_t)ch->n_rows * 4, kWsAlign);
    // (of the drafts' logits too, whether there are any or not; and shaped for more rows than there are where most of the
    // sequences have none: each adds its workgroups to the launches)
    const int64_t items = 2 * (int64_t)n_seqs * pl.max_new;
    pl.scan = scan_plan(std::max(std::min<int64_t>(items, 2 * (int64_t)ch->n_rows), items >> 13), 2 * (int64_t)ch->n_rows, vocab, dtype);
    pl.token = pl.scan.total;
    pl.logprob = pl.token + rows;
    pl.yes = pl.logprob + rows;
    pl.known = pl.yes + rows;
    pl.total = pl.known + align_up(2 * (size_t)ch->n_rows * sizeof(Known), kWsAlign);
    return MSAO_OK;
}

int run_scan(const void* a, void* s, void* e0, void* e1) { return launch_scan(*(const SampleArgs*)a, s, e0, e1); }
int run_verify_scan(const void* a, void* s, void* e0, void* e1) { return launch_verify_scan(*(const VerifyArgs*)a, s, e0, e1); }
int run_sample(const void* a, void* s, void* e0, void* e1) { return launch_sample(*(const SampleArgs*)a, s, e0, e1); }
int run_distribute(const void* a, void* s, void* e0, void* e1) { return launch_distribute(*(const VerifyArgs*)a, s, e0, e1); }
int run_verify_sums(const void* a, void* s, void* e0, void* e1) { return launch_verify_sums(*(const VerifyArgs*)a, s, e0, e1); }
int run_verify(const void* a, void* s, void* e0, void* e1) { return launch_verify(*(const VerifyArgs*)a, s, e0, e1); }
int run_join(const void* a, void* s, void* e0, void* e1) { return launch_verify_join(*(const VerifyArgs*)a, s, e0, e1); }

msao_status round_launch(msao_ctx* ctx, int kernel, void* stream, int (*fn)(const void*, void*, void*, void*), const void* a)
{
    return launched_in(ctx, ctx->round_rec[kernel], (hipStream_t)stream, fn, a);
}

// A kernel of `workgroups` workgroups of `threads` threads, in as many launches as that takes.
template <typename A>
msao_status row_launches(msao_ctx* ctx, int kernel, void* stream, int (*fn)(const void*, void*, void*, void*), A& a, int64_t workgroups, int threads)
{
    return (msao_status)in_launches(workgroups, threads, [&](int64_t first, int64_t n) -> int {
        a.first = (int32_t)first;
        a.blocks = (int32_t)n;
        return round_launch(ctx, kernel, stream, fn, &a);
    });
}

}  // namespace

extern "C" {

msao_status msao_sample_workspace(int64_t rows, int64_t vocab, int dtype, size_t* bytes)
{
    return guarded([&]() -> msao_status {
        if (!bytes) return bad(&g_err, "bytes is NULL");
        MSAO_TRY(check_rows_count(rows, &g_err));
        MSAO_TRY(check_vocab(vocab, dtype, &g_err));
        const ScanPlan pl = scan_plan(rows, rows, vocab, dtype);
        *bytes = pl.total;
        return MSAO_OK;
    });
}

msao_status msao_sample(msao_ctx* ctx, const void* logits, int64_t rows, int64_t vocab, int64_t row_stride, int dtype,
                        const msao_sampling* set, const float* u, const msao_sample_out* out, void* workspace,
                        size_t workspace_bytes, void* stream)
{
    return guarded([&]() -> msao_status {
        std::string* err = ctx ? &ctx->err : &g_err;
        MSAO_TRY(check_rows_count(rows, err));
        MSAO_TRY(check_vocab(vocab, dtype, err));
        MSAO_TRY(check_logits(logits, rows, vocab, row_stride, dtype, "logits", err));
        SampleArgs a;
        std::memset(&a, 0, sizeof a);
        MSAO_TRY(check_set(set, a.set, err));
        if (!out) return bad(err, "out is NULL");
        if (rows > 0 && !u) return bad(err, "u is NULL");
        MSAO_TRY(check_words({u, out->token, out->logprob, out->kept}, err));
        const ScanPlan pl = scan_plan(rows, rows, vocab, dtype);
        MSAO_TRY(check_workspace(workspace, workspace_bytes, pl.total, err));
        if (!ctx) return bad(err, "ctx is NULL");
        if (rows == 0) return MSAO_OK;
        a.logits = LogitRows{(const uint8_t*)logits, row_stride * elt_size(dtype)};
        a.u = u;
        a.rows = (int32_t)rows;
        a.vocab = (int32_t)vocab;
        a.dtype = dtype;
        a.token = out->token;
        a.logprob = out->logprob;
        a.kept = out->kept;
        a.scan = scan_at(pl, (uint8_t*)workspace);
        DeviceGuard guard(ctx->device);
        MSAO_TRY(round_launch(ctx, MSAO_ROUND_KERNEL_SCAN, stream, run_scan, &a));
        return row_launches(ctx, MSAO_ROUND_KERNEL_SAMPLE, stream, run_sample, a, rows, kRowThreads);
    });
}

msao_status msao_verify_workspace(const msao_chunk* chunk, int32_t n_seqs, int64_t vocab, int dtype, size_t* bytes)
{
    return guarded([&]() -> msao_status {
        if (!bytes) return bad(&g_err, "bytes is NULL");
        VerifyPlan pl;
        MSAO_TRY(verify_plan(chunk, n_seqs, vocab, dtype, pl, &g_err));
        *bytes = pl.total;
        return MSAO_OK;
    });
}

msao_status msao_verify(msao_ctx* ctx, const msao_chunk* chunk, int32_t n_seqs, const int32_t* tokens, const void* logits,
                        const void* draft_logits, int64_t vocab, int64_t row_stride, int64_t draft_stride, int dtype,
                        const msao_sampling* set, const float* u_accept, const float* u, const int32_t* length,
                        const msao_verify_out* out, void* workspace, size_t workspace_bytes, void* stream)
{
    return guarded([&]() -> msao_status {
        std::string* err = ctx ? &ctx->err : &g_err;
        VerifyPlan pl;
        MSAO_TRY(verify_plan(chunk, n_seqs, vocab, dtype, pl, err));
        if (n_seqs > 0 && !chunk->start) return bad(err, "start is NULL");
        MSAO_TRY(check_logits(logits, chunk->n_rows, vocab, row_stride, dtype, "logits", err));
        if (draft_logits) MSAO_TRY(check_logits(draft_logits, chunk->n_rows, vocab, draft_stride, dtype, "draft_logits", err));
        VerifyArgs a;
        std::memset(&a, 0, sizeof a);
        MSAO_TRY(check_set(set, a.set, err));
        if (!out) return bad(err, "out is NULL");
        if (chunk->n_rows > 0 && (!tokens || !u_accept || !u)) return bad(err, "tokens, u_accept or u is NULL");
        if (out->length && n_seqs > 0 && !length) return bad(err, "length is NULL");
        MSAO_TRY(check_words({chunk->start, tokens, u_accept, u, length, out->accepted, out->next, out->logprob, out->length}, err));
        MSAO_TRY(check_workspace(workspace, workspace_bytes, pl.total, err));
        if (!ctx) return bad(err, "ctx is NULL");
        if (n_seqs == 0) return MSAO_OK;
        const int64_t es = elt_size(dtype);
        a.logits = LogitRows{(const uint8_t*)logits, row_stride * es};
        a.draft = LogitRows{(const uint8_t*)draft_logits, draft_stride * es};
        a.ch = ChunkDev{chunk->start, chunk->n_rows, pl.max_new};
        a.n_seqs = n_seqs;
        a.vocab = (int32_t)vocab;
        a.dtype = dtype;
        a.tokens = tokens;
        a.u_accept = u_accept;
        a.u = u;
        a.length = length;
        a.accepted = out->accepted;
        a.next = out->next;
        a.logprob = out->logprob;
        a.length_out = out->length;
        uint8_t* ws = (uint8_t*)workspace;
        a.row_token = (int32_t*)(ws + pl.token);
        a.row_logprob = (float*)(ws + pl.logprob);
        a.row_yes = (int32_t*)(ws + pl.yes);
        a.known = (Known*)(ws + pl.known);
        a.scan = scan_at(pl.scan, ws);
        DeviceGuard guard(ctx->device);
        const int64_t pairs = (int64_t)n_seqs * pl.max_new, both = draft_logits ? 2 * pairs : pairs;
        MSAO_TRY(row_launches(ctx, MSAO_ROUND_KERNEL_SCAN, stream, run_verify_scan, a, both * a.scan.parts, kScanThreads));
        MSAO_TRY(row_launches(ctx, MSAO_ROUND_KERNEL_DISTRIBUTE, stream, run_distribute, a, both, kRowThreads));
        MSAO_TRY(round_launch(ctx, MSAO_ROUND_KERNEL_VERIFY_SUMS, stream, run_verify_sums, &a));
        MSAO_TRY(row_launches(ctx, MSAO_ROUND_KERNEL_VERIFY, stream, run_verify, a, pairs, kRowThreads));
        return round_launch(ctx, MSAO_ROUND_KERNEL_VERIFY_JOIN, stream, run_join, &a);
    });
}

msao_status msao_round_kernel_times(msao_ctx* ctx, float* ms)
{
    return guarded([&]() -> msao_status {
        if (!ctx || !ms) return MSAO_ERR_INVALID_ARG;
        return mean_times(ctx, ctx->round_rec, MSAO_NUM_ROUND_KERNELS, ms);
    });
}

}  // extern "C"
