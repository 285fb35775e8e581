// msao_cache_host.cpp -- host side of the paged cache's entry points: checks of
// arguments before anything is enqueued, launch shapes, workspaces.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <string>

#include "../../include/msao.h"
#include "msao_cache.h"
#include "msao_ctx.h"
#include "msao_internal.h"

using namespace msao;

namespace {

constexpr int64_t kMaxCapacity = (int64_t)1 << 29;
constexpr int64_t kMaxTokBytes = (int64_t)1 << 26;  // 16 tokens are one buffer
constexpr int64_t kMaxRowBytes = (int64_t)1 << 25;  // 64 rows' offsets stay in 31 bits
constexpr int64_t kMaxBlocks = (1 << 24) - 1;        // of 256 threads: a launch has fewer than 2^32
constexpr int64_t kMaxStride = (int64_t)1 << 40;    // elements; products with 31-bit counts stay in 63 bits with 2^10 pages to spare

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

msao_status check_strides(const int64_t* st, const msao_kv_cache& c, std::string* err)
{
    const int64_t es = elt_size(c.dtype);
    for (int i = 0; i < 3; ++i) {
        if (st[i] < 0 || st[i] > kMaxStride) return bad(err, "a cache stride is out of range");
        if (st[i] * es % 16 != 0) return fail(err, MSAO_ERR_ALIGNMENT, "a cache stride is not a multiple of 16 bytes");
    }
    if (st[2] < c.head_dim) return bad(err, "a token's stride is less than head_dim");
    if (st[2] * es >= kMaxTokBytes) return fail(err, MSAO_ERR_UNSUPPORTED, "a token's stride is 64 MiB or more");
    if (c.n_pages > 0 && st[0] > INT64_MAX / 8 / c.n_pages) return bad(err, "the page stride is out of range");
    return MSAO_OK;
}

msao_status check_cache(const msao_kv_cache* cache, std::string* err)
{
    if (!cache) return bad(err, "cache is NULL");
    const msao_kv_cache& c = *cache;
    if (c.dtype != MSAO_F32 && c.dtype != MSAO_BF16) return bad(err, "unknown dtype");
    if (c.head_dim < 8 || c.head_dim > MSAO_MAX_HEAD_DIM || c.head_dim % 8 != 0)
        return bad(err, "head_dim must be a multiple of 8, 8 .. 256");
    if (c.kv_heads < 1 || c.kv_heads > 65535) return bad(err, "kv_heads out of range");
    if (c.page_size < 16 || c.page_size > 65536 || (c.page_size & (c.page_size - 1)) != 0)
        return bad(err, "page_size must be a power of two, 16 .. 65536");
    if (c.n_pages < 0 || c.n_seqs < 0 || c.pages_per_seq < 0) return bad(err, "a count is negative");
    if ((int64_t)c.pages_per_seq * c.page_size > kMaxCapacity)
        return fail(err, MSAO_ERR_UNSUPPORTED, "a capacity of more than 2^29 tokens");
    if (c.table_stride < c.pages_per_seq) return bad(err, "table_stride < pages_per_seq");
    if (c.table_stride > kMaxStride || c.weight_stride > kMaxStride) return bad(err, "a stride is out of range");
    MSAO_TRY(check_strides(c.k_stride, c, err));
    MSAO_TRY(check_strides(c.v_stride, c, err));
    if (c.n_pages > 0 && (!c.k || !c.v)) return bad(err, "k or v is NULL");
    if (c.n_seqs > 0 && (!c.length || (c.pages_per_seq > 0 && !c.pages))) return bad(err, "pages or length is NULL");
    if (!aligned(c.k, 16) || !aligned(c.v, 16)) return fail(err, MSAO_ERR_ALIGNMENT, "k or v is not 16-byte aligned");
    if (!aligned(c.pages, 4) || !aligned(c.length, 4) || !aligned(c.weight, 4))
        return fail(err, MSAO_ERR_ALIGNMENT, "pages, length or weight is not 4-byte aligned");
    if (c.weight && c.weight_stride < (int64_t)c.pages_per_seq * c.page_size) return bad(err, "weight_stride < capacity");
    return MSAO_OK;
}

// Whether the cache can hold a token at all (an array of none may be NULL).
bool has_tokens(const msao_kv_cache& c) { return c.n_seqs > 0 && c.pages_per_seq > 0; }

msao_status check_chunk(const msao_chunk* ch, const msao_kv_cache& c, std::string* err)
{
    if (!ch) return bad(err, "chunk is NULL");
    if (ch->n_rows < 0) return bad(err, "n_rows is negative");
    if (ch->max_new < 0) return bad(err, "max_new is negative");
    if (c.n_seqs > 0 && !ch->start) return bad(err, "start is NULL");
    if (!aligned(ch->start, 4)) return fail(err, MSAO_ERR_ALIGNMENT, "start is not 4-byte aligned");
    return MSAO_OK;
}

// Rows of `values` values each: pointer, and the stride between them.
msao_status check_rows(const void* p, int64_t stride, int64_t values, int64_t es, const char* name, std::string* err)
{
    if (!p) return fail(err, MSAO_ERR_INVALID_ARG, std::string(name) + " is NULL");
    if (stride < values || stride > kMaxStride) return fail(err, MSAO_ERR_INVALID_ARG, std::string("the stride of ") + name + " is out of range");
    if (!aligned(p, 16) || stride * es % 16 != 0)
        return fail(err, MSAO_ERR_ALIGNMENT, std::string(name) + " or its stride is not a multiple of 16 bytes");
    return MSAO_OK;
}

msao_status check_heads(int heads, const msao_kv_cache& c, const msao_chunk& ch, std::string* err)
{
    if (heads < 1 || heads % c.kv_heads != 0) return bad(err, "heads must be a positive multiple of kv_heads");
    if ((int64_t)heads * std::max(ch.n_rows, 1) > INT32_MAX) return fail(err, MSAO_ERR_UNSUPPORTED, "2^31 rows of heads or more");
    return MSAO_OK;
}

msao_status check_append(const msao_kv_cache& c, const msao_chunk& ch, const msao_append* in, std::string* err)
{
    if (!in) return bad(err, "in is NULL");
    const int64_t es = elt_size(c.dtype), dim = c.head_dim;
    if (in->flags & ~MSAO_APPEND_NEIGHBOURS) return bad(err, "unknown flag bits");
    if (in->heads < 0 || in->heads > 65535) return bad(err, "heads out of range");
    if (ch.n_rows > 0) {
        if (in->heads > 0) {
            MSAO_TRY(check_rows(in->q, in->q_stride, in->heads * dim, es, "q", err));
            MSAO_TRY(check_rows(in->q_out, in->q_out_stride, in->heads * dim, es, "q_out", err));
            const bool in_place = in->q == in->q_out && (in->q_stride == in->q_out_stride || ch.n_rows == 1);
            if (!in_place && rows_meet(in->q, in->q_stride * es, in->q_out, in->q_out_stride * es, in->heads * dim * es, ch.n_rows))
                return bad(err, "q_out overlaps q and is not q");
        }
        MSAO_TRY(check_rows(in->k, in->k_stride, c.kv_heads * dim, es, "k", err));
        MSAO_TRY(check_rows(in->v, in->v_stride, c.kv_heads * dim, es, "v", err));
    }
    if (!aligned(in->q_norm, 16) || !aligned(in->k_norm, 16))
        return fail(err, MSAO_ERR_ALIGNMENT, "a norm's weight is not 16-byte aligned");
    if (!(in->eps >= 0.0f) || std::isinf(in->eps)) return bad(err, "eps must be finite and >= 0");
    if (in->rot_dim < 0 || in->rot_dim % 16 != 0 || in->rot_dim > dim)
        return bad(err, "rot_dim must be a multiple of 16, at most head_dim");
    if (in->rot_dim == 0) return MSAO_OK;
    if (!in->inv_freq) return bad(err, "inv_freq is NULL");
    if (in->n_axes < 1 || in->n_axes > MSAO_MAX_AXES) return bad(err, "n_axes must be 1 .. 4");
    if (!in->positions && in->n_axes != 1) return bad(err, "positions of several axes are NULL");
    if (in->positions && (in->position_stride < ch.n_rows || in->position_stride > kMaxStride))
        return bad(err, "position_stride < n_rows");
    if (!aligned(in->inv_freq, 4) || !aligned(in->positions, 4))
        return fail(err, MSAO_ERR_ALIGNMENT, "inv_freq or positions is not 4-byte aligned");
    int64_t pairs = 0;
    for (int i = 0; i < in->n_axes; ++i) {
        if (in->sections[i] < 0) return bad(err, "a section is negative");
        pairs += in->sections[i];
    }
    if (pairs != in->rot_dim / 2) return bad(err, "the sections do not sum to rot_dim / 2");
    return MSAO_OK;
}

int shift_of(int pow2)
{
    int s = 0;
    while (1 << s < pow2) ++s;
    return s;
}

CacheDev cache_dev(const msao_kv_cache& c)
{
    const int64_t es = elt_size(c.dtype);
    CacheDev d;
    std::memset(&d, 0, sizeof d);
    d.k = (uint8_t*)c.k;
    d.v = (uint8_t*)c.v;
    d.k_page = c.k_stride[0] * es;
    d.k_head = c.k_stride[1] * es;
    d.k_tok = c.k_stride[2] * es;
    d.v_page = c.v_stride[0] * es;
    d.v_head = c.v_stride[1] * es;
    d.v_tok = c.v_stride[2] * es;
    d.dim = c.head_dim;
    d.kv_heads = c.kv_heads;
    d.page_shift = shift_of(c.page_size);
    d.n_pages = c.n_pages;
    d.n_seqs = c.n_seqs;
    d.per_seq = c.pages_per_seq;
    d.table_stride = c.table_stride;
    d.pages = c.pages;
    d.length = c.length;
    d.weight = c.weight;
    d.weight_stride = c.weight_stride;
    return d;
}

ChunkDev chunk_dev(const msao_chunk& ch) { return ChunkDev{ch.start, ch.n_rows, std::min(ch.max_new, ch.n_rows)}; }

// The launch shape and the workspace of an attention call.
struct AttendPlan {
    AttendArgs a;
    size_t part_o, part_ml, lse2, part_w, total;
};
msao_status attend_plan(const msao_kv_cache* cache, const msao_chunk* chunk, int heads, uint32_t flags, AttendPlan& pl,
                        std::string* err)
{
    MSAO_TRY(check_cache(cache, err));
    MSAO_TRY(check_chunk(chunk, *cache, err));
    MSAO_TRY(check_heads(heads, *cache, *chunk, err));
    if (flags & ~(MSAO_ATTEND_CAUSAL | MSAO_ATTEND_WEIGHT)) return bad(err, "unknown flag bits");
    if ((flags & MSAO_ATTEND_WEIGHT) && !cache->weight && has_tokens(*cache)) return bad(err, "the cache has no weight to add to");
    AttendArgs& a = pl.a;
    std::memset(&a, 0, sizeof a);
    a.c = cache_dev(*cache);
    a.ch = chunk_dev(*chunk);
    a.heads = heads;
    a.group = make_group(heads / cache->kv_heads);
    a.dtype = cache->dtype;
    a.causal = flags & MSAO_ATTEND_CAUSAL ? 1 : 0;
    a.add_weight = flags & MSAO_ATTEND_WEIGHT ? 1 : 0;
    const int64_t groups = (int64_t)a.c.n_seqs * a.c.kv_heads;
    // (before the shape, whose products of counts would pass 63 bits)
    if (groups > kMaxBlocks) return fail(err, MSAO_ERR_UNSUPPORTED, "more workgroups than one launch takes");
    attend_shape(a);
    const AttendBlocks n = attend_blocks(a);
    const int64_t most = std::max(std::max(n.attend, n.combine), std::max(n.weight, n.join));
    if (groups > 0 && most > kMaxBlocks / groups) return fail(err, MSAO_ERR_UNSUPPORTED, "more workgroups than one launch takes");
    const AttendBytes b = attend_bytes(a);
    pl.part_o = 0;
    pl.part_ml = align_up(b.part_o, kWsAlign);
    pl.lse2 = pl.part_ml + align_up(b.part_ml, kWsAlign);
    pl.part_w = pl.lse2 + align_up(b.lse2, kWsAlign);
    pl.total = pl.part_w + align_up(b.part_w, kWsAlign);
    return MSAO_OK;
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

int run_append(const void* a, void* s, void* e0, void* e1) { return launch_append(*(const AppendArgs*)a, s, e0, e1); }
int run_attend(const void* a, void* s, void* e0, void* e1) { return launch_attend(*(const AttendArgs*)a, s, e0, e1); }
int run_combine(const void* a, void* s, void* e0, void* e1) { return launch_combine(*(const AttendArgs*)a, s, e0, e1); }
int run_weight(const void* a, void* s, void* e0, void* e1) { return launch_weight(*(const AttendArgs*)a, s, e0, e1); }
int run_weight_join(const void* a, void* s, void* e0, void* e1) { return launch_weight_join(*(const AttendArgs*)a, s, e0, e1); }
int run_select(const void* a, void* s, void* e0, void* e1) { return launch_select(*(const EvictArgs*)a, s, e0, e1); }
int run_move(const void* a, void* s, void* e0, void* e1) { return launch_move(*(const EvictArgs*)a, s, e0, e1); }

msao_status cache_launch(msao_ctx* ctx, int kernel, void* stream, int (*fn)(const void*, void*, void*, void*), const void* a)
{
    return launched_in(ctx, ctx->cache_rec[kernel], (hipStream_t)stream, fn, a);
}

}  // namespace

extern "C" {

msao_status msao_cache_validate(const msao_kv_cache* cache, const msao_chunk* chunk)
{
    return guarded([&] {
        MSAO_TRY(check_cache(cache, &g_err));
        return chunk ? check_chunk(chunk, *cache, &g_err) : MSAO_OK;
    });
}

msao_status msao_cache_append(msao_ctx* ctx, const msao_kv_cache* cache, const msao_chunk* chunk, const msao_append* in,
                              void* stream)
{
    return guarded([&]() -> msao_status {
        // (without a context the arguments are checked all the same)
        std::string* err = ctx ? &ctx->err : &g_err;
        MSAO_TRY(check_cache(cache, err));
        MSAO_TRY(check_chunk(chunk, *cache, err));
        MSAO_TRY(check_append(*cache, *chunk, in, err));
        if (!ctx) return bad(err, "ctx is NULL");
        if (chunk->n_rows == 0 || cache->n_seqs == 0) return MSAO_OK;
        AppendArgs a;
        std::memset(&a, 0, sizeof a);
        const int64_t es = elt_size(cache->dtype);
        a.c = cache_dev(*cache);
        a.ch = chunk_dev(*chunk);
        a.q = (const uint8_t*)in->q;
        a.q_out = (uint8_t*)in->q_out;
        a.k = (const uint8_t*)in->k;
        a.v = (const uint8_t*)in->v;
        a.q_stride = in->q_stride * es;
        a.q_out_stride = in->q_out_stride * es;
        a.k_stride = in->k_stride * es;
        a.v_stride = in->v_stride * es;
        a.q_norm = (const uint8_t*)in->q_norm;
        a.k_norm = (const uint8_t*)in->k_norm;
        a.eps = in->eps;
        a.heads = in->heads;
        a.rot = in->rot_dim;
        a.neighbours = in->flags & MSAO_APPEND_NEIGHBOURS ? 1 : 0;
        a.inv_freq = in->inv_freq;
        a.positions = in->positions;
        a.position_stride = in->position_stride;
        for (int i = 0, end = 0; i < 4; ++i) {
            if (a.rot > 0 && i < in->n_axes) end += in->sections[i];
            a.axis_end[i] = i < in->n_axes - 1 ? end : a.rot / 2;
        }
        a.dtype = cache->dtype;
        append_shape(a);
        if ((int64_t)a.ch.n_rows * a.parts > 4 * kMaxBlocks) return fail(err, MSAO_ERR_UNSUPPORTED, "more workgroups than one launch takes");
        DeviceGuard guard(ctx->device);
        return cache_launch(ctx, MSAO_CACHE_KERNEL_APPEND, stream, run_append, &a);
    });
}

msao_status msao_cache_attention_workspace(const msao_kv_cache* cache, const msao_chunk* chunk, int heads, uint32_t flags,
                                           size_t* bytes)
{
    return guarded([&]() -> msao_status {
        if (!bytes) return bad(&g_err, "bytes is NULL");
        AttendPlan pl;
        MSAO_TRY(attend_plan(cache, chunk, heads, flags, pl, &g_err));
        *bytes = pl.total;
        return MSAO_OK;
    });
}

msao_status msao_cache_attention(msao_ctx* ctx, const msao_kv_cache* cache, const msao_chunk* chunk, const void* q,
                                 int64_t q_stride, int heads, float scale, uint32_t flags, void* out, int64_t out_stride,
                                 float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    return guarded([&]() -> msao_status {
        std::string* err = ctx ? &ctx->err : &g_err;
        AttendPlan pl;
        MSAO_TRY(attend_plan(cache, chunk, heads, flags, pl, err));
        AttendArgs& a = pl.a;
        const int64_t es = elt_size(cache->dtype), values = (int64_t)heads * cache->head_dim;
        // (in base 2, as the kernels take it, too)
        const float scale2 = (float)((double)scale * 1.44269504088896340736);
        if (!std::isfinite(scale2)) return bad(err, "scale is not finite");
        if (chunk->n_rows > 0) {
            MSAO_TRY(check_rows(q, q_stride, values, es, "q", err));
            if (q_stride * es >= kMaxRowBytes) return fail(err, MSAO_ERR_UNSUPPORTED, "a stride of q of 32 MiB or more");
            MSAO_TRY(check_rows(out, out_stride, values, es, "out", err));
        }
        if (!aligned(lse, 4)) return fail(err, MSAO_ERR_ALIGNMENT, "lse is not 4-byte aligned");
        MSAO_TRY(check_workspace(workspace, workspace_bytes, pl.total, err));
        if (!ctx) return bad(err, "ctx is NULL");
        if (rows_meet(q, q_stride * es, out, out_stride * es, values * es, chunk->n_rows)) return bad(err, "out overlaps q");
        if (chunk->max_new == 0 || cache->n_seqs == 0) return MSAO_OK;
        a.q = (const uint8_t*)q;
        a.out = (uint8_t*)out;
        a.q_stride = q_stride * es;
        a.out_stride = out_stride * es;
        a.lse = lse;
        a.scale = scale2;
        uint8_t* ws = (uint8_t*)workspace;
        if (a.splits > 1) {
            a.part_o = (float*)(ws + pl.part_o);
            a.part_ml = (float*)(ws + pl.part_ml);
        }
        if (a.add_weight) {
            a.lse2 = (float*)(ws + pl.lse2);
            a.part_w = (float*)(ws + pl.part_w);
        }
        DeviceGuard guard(ctx->device);
        MSAO_TRY(cache_launch(ctx, MSAO_CACHE_KERNEL_ATTEND, stream, run_attend, &a));
        MSAO_TRY(cache_launch(ctx, MSAO_CACHE_KERNEL_COMBINE, stream, run_combine, &a));
        MSAO_TRY(cache_launch(ctx, MSAO_CACHE_KERNEL_WEIGHT, stream, run_weight, &a));
        return cache_launch(ctx, MSAO_CACHE_KERNEL_WEIGHT_JOIN, stream, run_weight_join, &a);
    });
}

msao_status msao_cache_evict_workspace(const msao_kv_cache* from, size_t* bytes)
{
    return guarded([&]() -> msao_status {
        if (!bytes) return bad(&g_err, "bytes is NULL");
        MSAO_TRY(check_cache(from, &g_err));
        *bytes = align_up((size_t)from->n_seqs * (size_t)from->kv_heads * sizeof(EvictInfo), kWsAlign);
        return MSAO_OK;
    });
}

msao_status msao_cache_evict(msao_ctx* ctx, const msao_kv_cache* from, const msao_kv_cache* to, const int32_t* budget,
                             int n_first, int n_recent, int32_t* kept_idx, int64_t idx_stride, void* workspace,
                             size_t workspace_bytes, void* stream)
{
    return guarded([&]() -> msao_status {
        std::string* err = ctx ? &ctx->err : &g_err;
        MSAO_TRY(check_cache(from, err));
        if (!from->weight && has_tokens(*from)) return bad(err, "the cache has no weight to evict by");
        const msao_kv_cache& dst = to ? *to : *from;
        if (to) {
            MSAO_TRY(check_cache(to, err));
            if (to->dtype != from->dtype || to->head_dim != from->head_dim || to->kv_heads != from->kv_heads ||
                to->n_seqs != from->n_seqs)
                return bad(err, "the caches differ in dtype, head_dim, kv_heads or n_seqs");
            // pages of one pool are told apart by their tables, on the device; arrays of
            // the same address are the same cache, whose moves need the order of `to` NULL
            if ((to->pages && to->pages == from->pages) || (to->length && to->length == from->length) ||
                (to->weight && to->weight == from->weight))
                return bad(err, "the caches share an array: pass NULL for eviction in place");
        }
        if (n_first < 0 || n_recent < 0) return bad(err, "n_first or n_recent is negative");
        const int64_t cap = (int64_t)from->pages_per_seq * from->page_size;
        if (from->n_seqs > 0 && !budget) return bad(err, "budget is NULL");
        if (from->n_seqs > 0 && cap > 0 && !kept_idx) return bad(err, "kept_idx is NULL");
        if (idx_stride < cap || idx_stride > kMaxStride) return bad(err, "idx_stride < capacity");
        if (!aligned(budget, 4) || !aligned(kept_idx, 4))
            return fail(err, MSAO_ERR_ALIGNMENT, "budget or kept_idx is not 4-byte aligned");
        EvictArgs a;
        std::memset(&a, 0, sizeof a);
        a.from = cache_dev(*from);
        a.to = cache_dev(dst);
        a.budget = budget;
        a.n_first = n_first;
        a.n_recent = n_recent;
        a.kept_idx = kept_idx;
        a.idx_stride = idx_stride;
        a.in_place = to ? 0 : 1;
        a.dtype = from->dtype;
        evict_shape(a);
        const int64_t groups = (int64_t)from->n_seqs * from->kv_heads * 2 * a.col_parts;
        // (the selection's workgroups have up to four times as many threads)
        if (groups > kMaxBlocks / std::max(a.blocks, 4)) return fail(err, MSAO_ERR_UNSUPPORTED, "more workgroups than one launch takes");
        size_t need = 0;
        MSAO_TRY(msao_cache_evict_workspace(from, &need));
        MSAO_TRY(check_workspace(workspace, workspace_bytes, need, err));
        if (!ctx) return bad(err, "ctx is NULL");
        if (from->n_seqs == 0) return MSAO_OK;
        a.info = (EvictInfo*)workspace;
        DeviceGuard guard(ctx->device);
        MSAO_TRY(cache_launch(ctx, MSAO_CACHE_KERNEL_SELECT, stream, run_select, &a));
        return cache_launch(ctx, MSAO_CACHE_KERNEL_MOVE, stream, run_move, &a);
    });
}

msao_status msao_cache_kernel_times(msao_ctx* ctx, float* ms)
{
    return guarded([&]() -> msao_status {
        if (!ctx || !ms) return MSAO_ERR_INVALID_ARG;
        return mean_times(ctx, ctx->cache_rec, MSAO_NUM_CACHE_KERNELS, ms);
    });
}

}  // extern "C"
