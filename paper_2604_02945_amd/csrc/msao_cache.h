// msao_cache.h -- the paged cache's kernels' arguments, and the indexing that
// kernels and host share: which rows a sequence has, where its tokens lie, how
// a row's tokens are cut into parts. Compiles for the host alone, so that the
// indexing is tested on the CPU (tests/c/cache_check.cpp). Not part of the ABI.
#pragma once

#include <stddef.h>
#include <stdint.h>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define MSAO_HD __host__ __device__ __forceinline__
#else
#define MSAO_HD inline
#endif

namespace msao {

// msao_kv_cache as the kernels take it: strides in bytes, the page size as a shift.
struct CacheDev {
    uint8_t* k;
    uint8_t* v;
    int64_t k_page, k_head, k_tok;
    int64_t v_page, v_head, v_tok;
    int32_t dim, kv_heads, page_shift, n_pages, n_seqs, per_seq;
    int64_t table_stride;
    const int32_t* pages;
    int32_t* length;
    float* weight;
    int64_t weight_stride;
};

struct ChunkDev {
    const int32_t* start;
    int32_t n_rows, max_new;
};

// An entry of a table that no kernel writes while it reads it: where the index is the same
// for a wavefront it comes through the scalar cache, and its wait is no wait for the vector
// loads before it.
MSAO_HD int entry(const int32_t* table, int64_t i)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)table)[i];
#else
    return table[i];
#endif
}

MSAO_HD int clamp_int(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

MSAO_HD int capacity(const CacheDev& c) { return c.per_seq << c.page_shift; }

// Tokens of sequence s, whatever the caller's array says.
MSAO_HD int seq_length(const CacheDev& c, int s) { return clamp_int(entry(c.length, s), 0, capacity(c)); }

// Rows of sequence s of the chunk: the first, and how many (all of them in [0, n_rows)).
struct Rows {
    int begin, n;
};
MSAO_HD Rows seq_rows(const ChunkDev& ch, int s)
{
    const int b = clamp_int(entry(ch.start, s), 0, ch.n_rows), e = clamp_int(entry(ch.start, s + 1), b, ch.n_rows);
    return Rows{b, e - b};
}

// The page that column `col` of the sequence's table names, -1 if it names none.
MSAO_HD int page_or_none(int page, int n_pages) { return page >= 0 && page < n_pages ? page : -1; }
MSAO_HD int page_at(const CacheDev& c, int s, int col)
{
    return page_or_none(entry(c.pages, (int64_t)s * c.table_stride + col), c.n_pages);
}

// How the `seen` tokens of a group of rows are cut: parts of `per` tokens (whole 32-token
// tiles; the last may be shorter), as many as it takes. No part for no token. Parts of
// one size, not a number of parts: sequences of any lengths give workgroups of equal work.
constexpr int kTile = 32;
MSAO_HD int parts_of(int seen, int per) { return seen <= 0 ? 0 : (seen - 1) / per + 1; }

// Query heads that share a kv head: row r of a (sequence, kv head) is query head r % n of token
// r / n. The quotient of a row in [0, 2^31) as the upper half of a product: with l the least of
// n <= 2^l and mul = floor(2^(31 + l) / n) + 1, r mul is r 2^(31 + l) / n and less than
// 2^(31 + l) / n more. (A division of integers is some 20 instructions, and there is one for each
// 16 bytes of queries: one prompt of 8,000 tokens, weight pass 412 us with it, 361 without.)
struct Group {
    int32_t n;
    uint32_t mul;
    int32_t shift;
    MSAO_HD int of(int row) const
    {
        return (int)((uint32_t)(((uint64_t)(2 * (uint32_t)row) * mul) >> 32) >> shift);
    }
};
MSAO_HD Group make_group(int n)
{
    Group g{n, 0, 0};
    while (g.shift < 31 && (int64_t)1 << g.shift < n) ++g.shift;
    const uint64_t mul = ((uint64_t)1 << (31 + g.shift)) / (uint32_t)n + 1;
    g.mul = (uint32_t)mul;
    return g;
}

// Tokens that rows [r0, r0 + rows) of a (sequence, kv head) see at most: row r is
// query head r % group.n of token r / group.n. Without `causal` all of them.
MSAO_HD int group_sees(int length, int n_new, const Group& group, int last_row, bool causal)
{
    return causal ? clamp_int(length - n_new + group.of(last_row) + 1, 0, length) : length;
}

// Whether n rows of `bytes` bytes from a, every `sa` bytes, and from b, every `sb` (both at
// least `bytes`), certainly share memory: exact for rows at one distance, which may lie between
// one another as the parts of one projection do; at different ones the first rows are compared.
MSAO_HD bool rows_meet(const void* a, int64_t sa, const void* b, int64_t sb, int64_t bytes, int64_t n)
{
    if (n <= 0) return false;
    const int64_t d = (int64_t)((uintptr_t)b - (uintptr_t)a);
    if (d > -bytes && d < bytes) return true;
    if (sa != sb) return false;
    const int64_t k = d / sa - (d % sa < 0 ? 1 : 0), r = d - k * sa;  // b's first row is r past the k-th of a, and sa - r before the next
    return (r < bytes && k > -n && k < n) || (sa - r < bytes && k + 1 > -n && k + 1 < n);
}

// ---- append -------------------------------------------------------------------
struct AppendArgs {
    CacheDev c;
    ChunkDev ch;
    const uint8_t* q;
    uint8_t* q_out;
    const uint8_t* k;
    const uint8_t* v;
    int64_t q_stride, q_out_stride, k_stride, v_stride;  // bytes
    const uint8_t* q_norm;
    const uint8_t* k_norm;
    float eps;
    int32_t heads, rot, neighbours;
    const float* inv_freq;
    const int32_t* positions;
    int64_t position_stride;
    int32_t axis_end[4];  // first pair past each axis
    int32_t dtype;
    int32_t lanes;        // lanes of a head
    int32_t parts;        // wavefronts of a token
};

// ---- attention ------------------------------------------------------------------
struct AttendArgs {
    CacheDev c;
    ChunkDev ch;
    const uint8_t* q;
    uint8_t* out;
    int64_t q_stride, out_stride;  // bytes
    float* lse;
    int32_t heads, dtype;
    Group group;
    int32_t causal, add_weight;
    float scale;                   // scale * log2(e)
    int32_t part_tokens;           // tokens of a part
    int32_t splits, row_tiles;     // most parts of a group of rows; groups of a (sequence, kv head)
    int32_t tile_rows;             // rows of a group
    int32_t weight_tokens;         // tokens of a part in the weight pass
    int32_t weight_parts;          // most of them for each (sequence, kv head)
    int32_t row_parts;             // and of the rows
    // workspace
    float* part_o;                 // [splits][n_rows * heads][dim], a part's sum of 2^(x - m) v
    float* part_ml;                // [splits][n_rows * heads][2], its m and sum of 2^(x - m)
    float* lse2;                   // [n_rows * heads] log2 of the sums, for the weight pass
    float* part_w;                 // [row_parts][n_seqs * kv_heads][capacity]
};

// ---- eviction -------------------------------------------------------------------
struct EvictInfo {
    int32_t kept, first_moved;     // tokens that stay; the first of them whose place changes
};
struct EvictArgs {
    CacheDev from, to;
    const int32_t* budget;
    int32_t n_first, n_recent;
    int32_t* kept_idx;
    int64_t idx_stride;
    EvictInfo* info;               // workspace [n_seqs * kv_heads]
    int32_t in_place, dtype;
    int32_t blocks;                // of the move, for each (sequence, kv head, k or v, column part)
    int32_t col_parts;             // parts that a row is cut into
    Group units;                   // 16-byte pieces of a row's part
};

int launch_append(const AppendArgs& a, void* stream, void* ev0, void* ev1);
int launch_attend(const AttendArgs& a, void* stream, void* ev0, void* ev1);
int launch_combine(const AttendArgs& a, void* stream, void* ev0, void* ev1);
int launch_weight(const AttendArgs& a, void* stream, void* ev0, void* ev1);
int launch_weight_join(const AttendArgs& a, void* stream, void* ev0, void* ev1);
int launch_select(const EvictArgs& a, void* stream, void* ev0, void* ev1);
int launch_move(const EvictArgs& a, void* stream, void* ev0, void* ev1);

// Launch shapes: lanes and parts of an append; blocks and col_parts of an eviction's move.
void append_shape(AppendArgs& a);
void evict_shape(EvictArgs& a);
// Launch shape of an attention call: fills part_tokens .. row_parts.
void attend_shape(AttendArgs& a);
// Workgroups that its kernels launch for each (sequence, kv head); 0: no such launch.
struct AttendBlocks {
    int64_t attend, combine, weight, join;
};
AttendBlocks attend_blocks(const AttendArgs& a);
// Bytes of each of its workspace arrays.
struct AttendBytes {
    size_t part_o, part_ml, lse2, part_w;
};
AttendBytes attend_bytes(const AttendArgs& a);

}  // namespace msao
