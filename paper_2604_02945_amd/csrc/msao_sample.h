// msao_sample.h -- arguments of the kernels that draw tokens from rows of logits and
// verify drafts against them. Not part of the ABI.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "msao_cache.h"

namespace msao {

// Rows of logits: row r starts at base + r * row_bytes.
struct LogitRows {
    const uint8_t* base;
    int64_t row_bytes;
};

// msao_sampling: per row, each may be NULL.
struct SamplingDev {
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
};

constexpr int64_t kMaxVocab = (int64_t)1 << 20;
constexpr int kRowThreads = 1024;   // of the kernels that have a workgroup a row,
constexpr int kScanThreads = 256;   // and of those with many workgroups a row

// Workgroups of `threads` threads in launches of fewer than 2^32 threads each, which is what one takes: f(first, how many) for
// each launch until one does not give 0.
template <typename F>
int in_launches(int64_t workgroups, int threads, F f)
{
    const int64_t most = (((int64_t)1 << 32) - 1) / threads;
    int rc = 0;
    for (int64_t at = 0; at < workgroups && rc == 0; at += most) rc = f(at, workgroups - at < most ? workgroups - at : most);
    return rc;
}

// What the rows' first reading leaves, row by row (a verification's drafts' logits behind the others). A segment
// is 64 loads of 16 bytes, a share `lanes` of them.
struct ScanDev {
    float* most;               // [rows][shares] the largest logit, NaN for what makes a row have no distribution
    double* sum;               // [rows][segments] the weights' sum relative to the segment's largest logit,
    float* of;                 // [rows][segments] which this is,
    int32_t* number;           // [rows][segments] and how many of them are above -inf
    int32_t lanes, shares, segments;
    int32_t per, parts;        // segments of a workgroup; workgroups of a row (0: rows are not read first)
};
struct RowScan {
    float* most;
    double* sum;
    float* of;
    int32_t* number;
};
MSAO_HD RowScan scan_of(const ScanDev& s, int64_t row)
{
    return RowScan{s.most + row * s.shares, s.sum + row * s.segments, s.of + row * s.segments, s.number + row * s.segments};
}
void scan_shape(ScanDev& d, int64_t rows, int64_t vocab, int dtype);

struct SampleArgs {
    LogitRows logits;
    SamplingDev set;
    const float* u;
    int32_t rows, vocab, dtype;
    int32_t first, blocks;     // workgroups of this launch
    int32_t* token;
    float* logprob;
    int32_t* kept;
    ScanDev scan;              // workspace
};

// Of a distribution what weighs a token in it.
struct Known {
    double m, inv, zero, least, total;
    float cut;
    int32_t cut_at, kept, best, none;
};

// Place of row r's distribution, or (`which` 1) of the draft's behind it, which lie behind all rows' ones: past 31 bits of
// more than 2^30 rows.
MSAO_HD int64_t dist_at(const ChunkDev& ch, int which, int r) { return (int64_t)which * ch.n_rows + r; }

struct VerifyArgs {
    LogitRows logits, draft;   // draft.base NULL: drafts are certain
    SamplingDev set;
    ChunkDev ch;
    int32_t n_seqs, vocab, dtype;
    int32_t first, blocks;     // workgroups of this launch
    const int32_t* tokens;
    const float* u_accept;
    const float* u;
    const int32_t* length;
    int32_t* accepted;
    int32_t* next;
    float* logprob;
    int32_t* length_out;
    // workspace [n_rows]
    int32_t* row_token;        // the token that follows the row
    float* row_logprob;
    int32_t* row_yes;          // whether it is the row's draft
    Known* known;              // [2 n_rows], the drafts' ones behind the rows'
    ScanDev scan;
};

int launch_scan(const SampleArgs& a, void* stream, void* ev0, void* ev1);
int launch_verify_scan(const VerifyArgs& a, void* stream, void* ev0, void* ev1);
int launch_sample(const SampleArgs& a, void* stream, void* ev0, void* ev1);
int launch_distribute(const VerifyArgs& a, void* stream, void* ev0, void* ev1);
int launch_verify_sums(const VerifyArgs& a, void* stream, void* ev0, void* ev1);
int launch_verify(const VerifyArgs& a, void* stream, void* ev0, void* ev1);
int launch_verify_join(const VerifyArgs& a, void* stream, void* ev0, void* ev1);

}  // namespace msao
