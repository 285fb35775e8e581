// msao_sample.hip -- gfx950 (CDNA4) kernels that draw a token from each row of logits and
// verify drafted tokens against such rows (Sec. 4.2).
//
// A row's distribution: w_v = 2^((x_v - max) log2(e) / T) over the tokens that stay, which
// are a head of the order (logit down, index up): the top_k first, of them the fewest whose
// weight is top_p of theirs, of them those with w >= min_p. A token is the first of its
// indices whose running sum passes u times the whole. Every comparison of sums is one of
// 64-bit weights and sums: in 32 bits sums over 10^5 tokens are off by more than the
// lightest token's weight, and the answer would be another token now and then.
//
// k_scan reads the rows, many workgroups a row, and leaves for each segment (a wavefront's 64 loads
// of 16 bytes) the largest logit, the largest of each share of it (1, 4 or 16 loads), and where every
// token may stay the sum of the weights relative to the segment's largest and their number. Then one workgroup of 1,024
// threads has a row (k_sample; of a verification k_distribute finds the distributions, k_verify_sums the sums of
// rows of which many tokens may be drawn, k_verify the tokens):
//  - without top_k, top_p and min_p the segments' sums say in which one the token lies;
//  - the head of the order is mostly short. The j-th largest of the shares' maxima is a bound
//    that j tokens at least reach and few more, and only shares whose maximum reaches it are
//    read again. Up to 1,024 such tokens are sorted;
//  - a longer head is found by 2,048 bins that are even in the logit, between the largest one and one
//    below which too little weight lies: 32-bit sums say which bins the head may end in, then
//    one reading sums the weights above them in 64 bits and collects the tokens in them, which
//    are ranked as above. That the head ends there is checked;
//  - where it does not, or the bins hold too many tokens (equal ones), bins of keys close in on its end.
// A weight is some ten instructions of 64 bits (a table of 256 and a polynomial of degree 3), which take two thirds of
// a summed row's time; any other row is bound by its reading.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "msao_device.h"
#include "msao_internal.h"
#include "msao_sample.h"

namespace msao {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;

constexpr int kWave = 64;
constexpr int kThreads = kRowThreads;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2 * kThreads;
constexpr int kList = kThreads;            // tokens that are ranked in LDS
// Of the shares' maxima, for a head whose length top_p decides: 256 rows with mixed settings 112 us in the row kernel, 106
// with 128 and 117 with 512 (more to rank, for few heads that are longer).
constexpr int kTryHead = 256;
// Workgroups of a scan: 64 requests' drafts 37 us, 47 with 1,024, 29 with 4,096; 256 rows 27, 31, 23.
constexpr int64_t kScanTarget = 2048;
constexpr int kScanWaves = kScanThreads / kWave, kScanAhead = 4;
constexpr double kMagic = 26388279066624.0;  // 1.5 2^44: a number added to it is rounded to 1 / 256, which is its last digit
constexpr double kLog2e = 1.4426950408889634074;
constexpr double kLn2 = 0.69314718055994530942;
constexpr double kSame = 0x1p-42;          // of a weight: no more than this is none (the weights' error; their sums' is less), so that
                                           // equal distributions have nothing between them, whichever way each was summed
constexpr int kMostSegments = 4096;        // of a row of kMaxVocab float32 logits
constexpr int kNone = 0x7FFFFFFF;

// Keys in the order of the values; +0 and -0 are one.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// a b + c with c in scalar registers: for a polynomial's constants the compiler takes the form that adds to its own
// operand, and a move of the constant with it.
__device__ __forceinline__ double fma_constant(double a, double b, double c)
{
    double r;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "s"(c));
    return r;
}

// 2^(d inv) for d of at most 0: 2^n times 2^(k / 256) from a table times a polynomial of degree 3 in the rest, which is
// within 1/512 of 0: off by (ln 2 / 512)^4 / 24, 1.4e-13 of the value, and by the table's 3.3e-14; equal logits
// have the weight 1. `least` is -1000 / inv: what lies below it, -inf too, gives 2^-1000. M at a time, so that no
// step waits for the one before it. A scan of 256 bf16 rows of 151,936 with sums takes 38 us, 16 without them (by a polynomial
// of degree 9 and no table 40): of 160 float32 rows' 35 us vector instructions are issued for 24, at four clocks a wavefront
// each, and the table's reads have bank conflicts for 3.
constexpr int kTable = 256;
template <int M>
__device__ __forceinline__ void exp2_of(const double* table, double (&d)[M], double inv, double least)
{
    double r[M], w[M];
    int n[M];
#pragma unroll
    for (int e = 0; e < M; ++e) {
        d[e] = fmax(d[e], least);
        const double t = fma(d[e], inv, kMagic);  // in its low word 256 d inv, rounded (an ulp is 1 / 256)
        r[e] = fma(d[e], inv, kMagic - t);
        n[e] = __double2loint(t);
        w[e] = table[n[e] & (kTable - 1)];
        d[e] = fma_constant(r[e], 0.05550410866482158, 0.24022650695910072);  // ln 2^3 / 6, ln 2^2 / 2
    }
#pragma unroll
    for (int e = 0; e < M; ++e) d[e] = fma_constant(d[e], r[e], 0.6931471805599453);
#pragma unroll
    for (int e = 0; e < M; ++e) {
        d[e] = fma(w[e] * r[e], d[e], w[e]);
        // (n of -1000 at least: added to the exponent)
        d[e] = __hiloint2double(__double2hiint(d[e]) + ((n[e] >> 8) << 20), __double2loint(d[e]));
    }
}
__device__ __forceinline__ double exp2_of(const double* table, double d, double inv, double least)
{
    double v[1] = {d};
    exp2_of(table, v, inv, least);
    return v[0];
}

// The table: 2^r by a polynomial, the interpolation of 2^r at Chebyshev's nodes in [-1/2, 1/2] with the first
// coefficient made 1, off by 3.3e-14.
__device__ __forceinline__ void fill_table(double* table)
{
    for (int k = threadIdx.x; k < kTable; k += blockDim.x) {
        const double r = (k < kTable / 2 ? k : k - kTable) * (1.0 / kTable);
        double p = 1.020869083593037e-07;
        p = fma(p, r, 1.3259646250270451e-06);
        p = fma(p, r, 1.5252657257186041e-05);
        p = fma(p, r, 0.00015403433746224196);
        p = fma(p, r, 0.0013333558230170627);
        p = fma(p, r, 0.009618129193942167);
        p = fma(p, r, 0.05550410866444768);
        p = fma(p, r, 0.240226506956403);
        p = fma(p, r, 0.69314718055995);
        p = fma(p, r, 1.0);
        table[k] = k < kTable / 2 ? p : 2.0 * p;
    }
    __syncthreads();
}

// log2(e) / T, of an infinite T not quite 0, so that the exponent of -inf is
// no product of 0 and an infinity.
__device__ __forceinline__ double inverse_of(float temperature) { return fmax(kLog2e / (double)temperature, 1e-300); }
constexpr double kLeast = -1000.0;  // exponents below it are no weight

// 16 bytes of a row, widened; what lies past its end, and -inf, is the value that no token has.
template <int DT>
struct Chunk {
    static constexpr int N = DT == kBF16 ? 8 : 4;
    float x[N];
    __device__ __forceinline__ explicit Chunk(const u32x4& w)
    {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if constexpr (DT == kBF16) x[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
            else x[e] = __uint_as_float(w[e]);
        }
    }
    __device__ __forceinline__ void end(int n)
    {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = e < n ? x[e] : -INFINITY;
    }
};

// A row of logits as a workgroup walks it: step i has thread t at the 16 bytes i * kThreads + t,
// so that (step, wavefront, lane) is the order of the indices. Segment i * kWaves + w is wavefront w's.
template <int DT>
struct Row {
    static constexpr int N = Chunk<DT>::N;
    rsrc_t r;
    int vocab, steps, segments;
    __device__ __forceinline__ Row(const LogitRows& rows, int64_t row, int vocab_) : vocab(vocab_)
    {
        constexpr int es = DT == kBF16 ? 2 : 4;
        // (whole words: a row's pitch is a multiple of 16 bytes)
        r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(rows.base) + row * rows.row_bytes, (short)0,
                                              (vocab * es + 3) & ~3, 0x00020000);
        const int chunks = (vocab + N - 1) / N;
        steps = (chunks + kThreads - 1) / kThreads;
        segments = (chunks + kWave - 1) / kWave;
    }
    __device__ __forceinline__ u32x4 load(int chunk) const { return __builtin_amdgcn_raw_buffer_load_b128(r, chunk * 16, 0, 0); }
    __device__ __forceinline__ Chunk<DT> at(int chunk) const
    {
        Chunk<DT> c(load(chunk));
        c.end(vocab - chunk * N);
        return c;
    }
    // f(step, first index, chunk) for every step, kAhead of which are loaded at a time (two where f takes many registers)
    template <int kAhead = 4, typename F>
    __device__ __forceinline__ void each(F f) const
    {
        const int t = threadIdx.x, wave_end = (uniform(t >> 6) + 1) * kWave;
#pragma unroll 1
        for (int i0 = 0; i0 < steps; i0 += kAhead) {
            u32x4 w[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) w[a] = load((i0 + a) * kThreads + t);
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int i = i0 + a, c = i * kThreads + t;
                if (i >= steps) break;
                Chunk<DT> x(w[a]);
                if ((i * kThreads + wave_end) * N > vocab) x.end(vocab - c * N);
                f(i, c * N, x);
            }
        }
    }
    __device__ __forceinline__ float value(int v) const
    {
        if constexpr (DT == kBF16) return __uint_as_float((uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, 2 * v, 0, 0) << 16);
        return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, 4 * v, 0, 0));
    }
};

// The settings of row r.
struct Settings {
    float temperature, top_p, min_p;
    int top_k;
    __device__ __forceinline__ bool greedy() const { return !(temperature > 0.0f); }
    __device__ __forceinline__ bool by_k(int vocab) const { return top_k > 0 && top_k < vocab; }
    // whether the sum over all tokens is needed
    __device__ __forceinline__ bool sums(int vocab) const { return !greedy() && !by_k(vocab) && (top_p < 1.0f || !(min_p > 0.0f)); }
};
__device__ __forceinline__ Settings settings_of(const SamplingDev& s, int r)
{
    return Settings{s.temperature ? s.temperature[r] : 1.0f, s.top_p ? s.top_p[r] : 1.0f, s.min_p ? s.min_p[r] : 0.0f,
                    s.top_k ? s.top_k[r] : 0};
}

// The lane's value with DPP control CTRL in the rows of ROWS, 0 where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)moved<CTRL, ROWS>((int)(uint32_t)b), hi = (uint32_t)moved<CTRL, ROWS>((int)(uint32_t)(b >> 32));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int CTRL>
__device__ __forceinline__ float turned(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}

// Sums of the lanes up to each: within rows of 16 lanes, then lane 15 of a row to the next row and
// lane 31 to the upper half.
template <typename T>
__device__ __forceinline__ T wave_scan(T v)
{
    v += moved<0x111, 0xF>(v);
    v += moved<0x112, 0xF>(v);
    v += moved<0x114, 0xF>(v);
    v += moved<0x118, 0xF>(v);
    v += moved<0x142, 0xA>(v);
    v += moved<0x143, 0xC>(v);
    return v;
}

// ---- the rows' first reading ---------------------------------------------------------

// Segments s, s + step, .. up to `end` of a row, by one wavefront.
template <int DT, int SHARE>
__device__ __forceinline__ void scan_segments(const double* table, const Row<DT>& row, const RowScan& scan, const Settings& set, int first, int step, int end)
{
    constexpr int N = Chunk<DT>::N;
    const int lane = threadIdx.x & (kWave - 1);
    const bool sums = set.sums(row.vocab);
    const double inv = inverse_of(set.temperature), least = kLeast / inv;
#pragma unroll 1
    for (int s0 = first; s0 < end; s0 += step * kScanAhead) {
        u32x4 w[kScanAhead];
#pragma unroll
        for (int a = 0; a < kScanAhead; ++a) w[a] = row.load(min(s0 + a * step, end - 1) * kWave + lane);
#pragma unroll
        for (int a = 0; a < kScanAhead; ++a) {
            const int s = s0 + a * step;
            if (s >= end) break;
            Chunk<DT> c(w[a]);
            if ((s + 1) * kWave * N > row.vocab) c.end(row.vocab - (s * kWave + lane) * N);
            bool bad = false;
            float m = c.x[0];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                bad = bad || !(c.x[e] < INFINITY);
                m = fmaxf(m, c.x[e]);
            }
            if (bad) m = __builtin_nanf("");  // (kept by the comparisons below, so that the row knows)
            auto join = [](float a, float b) { return a > b || !(a == a) ? a : b; };
            if (SHARE >= 4) {
                m = join(m, turned<0xB1>(m));  // lanes of four
                m = join(m, turned<0x4E>(m));
            }
            if (SHARE == 16) {
                m = join(m, turned<0x124>(m));  // rows of 16 turned by 4 and 8
                m = join(m, turned<0x128>(m));
            }
            if (lane % SHARE == 0) scan.most[s * (kWave / SHARE) + lane / SHARE] = m;
            if (!sums) continue;
            if (SHARE == 1) {
                m = join(m, turned<0xB1>(m));
                m = join(m, turned<0x4E>(m));
            }
            if (SHARE <= 4) {
                m = join(m, turned<0x124>(m));
                m = join(m, turned<0x128>(m));
            }
            m = join(m, __shfl_xor(m, 16));
            m = join(m, __shfl_xor(m, 32));
            // (the largest adds 1: what 2^-1000 of the others does not change)
            double sum = 0.0;
            int number = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) number += __popcll(__ballot(c.x[e] > -INFINITY));
            if (m > -INFINITY) {
#pragma unroll
                for (int h = 0; h < N; h += 4) {
                    double w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = (double)c.x[h + e] - (double)m;
                    exp2_of(table, w, inv, least);
                    sum += (w[0] + w[1]) + (w[2] + w[3]);
                }
            }
            sum = wave_scan(sum);
            if (lane == kWave - 1) {
                scan.sum[s] = sum;
                scan.of[s] = m;
                scan.number[s] = number;
            }
        }
    }
}

template <int DT, int SHARE>
__device__ __forceinline__ void scan_part(const LogitRows& rows, const ScanDev& scan, const SamplingDev& set, int vocab, int r, int64_t at, int part)
{
    __shared__ double table[kTable];
    const Row<DT> row(rows, r, vocab);
    const int wave = uniform(threadIdx.x >> 6), first = part * scan.per;
    const Settings mine = settings_of(set, r);
    if (mine.sums(vocab)) fill_table(table);
    scan_segments<DT, SHARE>(table, row, scan_of(scan, at), mine, first + wave, kScanWaves, min(first + scan.per, row.segments));
}

template <int DT, int SHARE>
__global__ __launch_bounds__(kScanThreads) void k_scan(SampleArgs a)
{
    const int r = blockIdx.x / a.scan.parts, part = blockIdx.x - r * a.scan.parts;
    scan_part<DT, SHARE>(a.logits, a.scan, a.set, a.vocab, r, r, part);
}

// Of a verification: the rows that it looks at, and the ones of the drafts' logits that it needs.
template <int DT, int SHARE>
__global__ __launch_bounds__(kScanThreads) void k_verify_scan(VerifyArgs a)
{
    const int block = a.first + (int)blockIdx.x, item = block / a.scan.parts, part = block - item * a.scan.parts;
    const int pairs = a.n_seqs * a.ch.max_new, which = item >= pairs ? 1 : 0, s = (item - which * pairs) / a.ch.max_new;
    const int i = item - which * pairs - s * a.ch.max_new;
    const Rows rows = seq_rows(a.ch, s);
    if (i >= min(rows.n, a.ch.max_new) - which) return;
    const int r = rows.begin + i;
    scan_part<DT, SHARE>(which ? a.draft : a.logits, a.scan, a.set, a.vocab, r, dist_at(a.ch, which, r), part);
}

// ---- one row ---------------------------------------------------------------------------

// Scratch that the steps of a row share.
struct Scratch {
    union {
        uint64_t mass[2][kBins];      // a bin's weight in units of 2^-43 and of 2^-86
        uint32_t count[kBins];
        double segment[kMostSegments];
    };
    uint64_t packed[kList];           // key, and the index' complement: the order of the tokens, upside down
    union {
        int share[kList];
        int order[kMostSegments];     // counts of segments
    };
    float list_x[kList];              // tokens that stay, by index
    int list_at[kList];
    double wave_d[2][kWaves];
    int wave_i[2][kWaves];
    float wave_f[2][kWaves];
    double table[kTable];             // 2^(k / 256)
    double found_d;
    int found_i[3];
    int n;
};

// A thread's view of it. Sums over the workgroup use two rooms in turn, so that one barrier each is enough: who
// writes a room again has passed the barrier of the sum between, and with it everybody has read.
struct Lds {
    Scratch& s;
    uint64_t (&mass)[2][kBins];
    uint32_t (&count)[kBins];
    double (&segment)[kMostSegments];
    uint64_t (&packed)[kList];
    int (&share)[kList];
    int (&order)[kMostSegments];
    float (&list_x)[kList];
    int (&list_at)[kList];
    double& found_d;
    int (&found_i)[3];
    int& n;
    int turn = 0;
    __device__ __forceinline__ explicit Lds(Scratch& r)
        : s(r), mass(r.mass), count(r.count), segment(r.segment), packed(r.packed), share(r.share),
          order(r.order), list_x(r.list_x), list_at(r.list_at), found_d(r.found_d), found_i(r.found_i), n(r.n)
    {
    }
    __device__ __forceinline__ double* room(double) { return s.wave_d[turn ^= 1]; }
    __device__ __forceinline__ int* room(int) { return s.wave_i[turn ^= 1]; }
};

// A row's distribution.
struct Dist {
    bool none;        // a NaN, +inf, or no finite logit
    bool listed;      // the tokens that stay are in lds.list, in the order of their indices
    bool summed;      // lds.segment has the sums of the weights
    int best;         // of a row whose largest logit alone stays, its index; else -1
    int kept;         // how many stay where that is known, else -1
    int n;            // entries of the list
    double m, inv;    // largest logit; log2(e) / T
    double zero;      // differences of logits below it have no weight
    float cut;        // tokens stay with a logit above it, or equal to it and an index up to cut_at,
    int cut_at;
    double least;     // and (x - m) inv of at least this
    double total;     // of the weights; known where `kept` is or `summed`
    const double* table;
    __device__ __forceinline__ double exponent(float x) const { return ((double)x - m) * inv; }
    __device__ __forceinline__ double power(float x) const
    {
        const double by = (double)x - m, p = exp2_of(table, by, inv, zero);
        return by >= zero ? p : 0.0;
    }
    __device__ __forceinline__ bool stays(float x, int v) const
    {
        return (x > cut || (x == cut && v <= cut_at)) && (least == -INFINITY || exponent(x) >= least);
    }
    __device__ __forceinline__ double weight(float x, int v) const { return stays(x, v) ? power(x) : 0.0; }
};

// Sum over the threads before this one, and the whole. All threads.
template <typename T>
__device__ __forceinline__ T block_before(T v, Lds& lds, T& total)
{
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    T* room = lds.room(T(0));
    const T upto = wave_scan(v);
    if (lane == kWave - 1) room[wave] = upto;
    __syncthreads();
    T before = 0;
    total = 0;
#pragma unroll 4
    for (int w = 0; w < kWaves; ++w) {
        const T s = room[w];
        before += w < wave ? s : T(0);
        total += s;
    }
    return before + (upto - v);
}

__device__ __forceinline__ double* segments_of(Lds& lds, double) { return lds.segment; }
__device__ __forceinline__ int* segments_of(Lds& lds, int) { return lds.order; }

// The sums of f(x, v) >= 0 over the row's segments, in the order of the indices.
template <typename T, int DT, typename F>
__device__ __forceinline__ void sum_segments(const Row<DT>& row, Lds& lds, F f)
{
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    T* segment = segments_of(lds, T(0));
    __syncthreads();
    row.template each<2>([&](int i, int v, const Chunk<DT>& c) {
        T s = 0;
#pragma unroll
        for (int e = 0; e < Row<DT>::N; ++e) s += f(c.x[e], v + e);
        s = wave_scan(s);
        if (lane == kWave - 1) segment[i * kWaves + wave] = s;
    });
    __syncthreads();
}

// Of f(x, y, v) with y the other row's logit.
template <typename T, int DT, typename F>
__device__ __forceinline__ void sum_segments(const Row<DT>& row, Lds& lds, const Row<DT>& other, F f)
{
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    T* segment = segments_of(lds, T(0));
    __syncthreads();
    row.template each<2>([&](int i, int v, const Chunk<DT>& c) {
        const Chunk<DT> o = other.at(i * kThreads + (int)threadIdx.x);
        T s = 0;
#pragma unroll
        for (int e = 0; e < Row<DT>::N; ++e) s += f(c.x[e], o.x[e], v + e);
        s = wave_scan(s);
        if (lane == kWave - 1) segment[i * kWaves + wave] = s;
    });
    __syncthreads();
}

__device__ __forceinline__ double sum_of_segments(Lds& lds, int segments)
{
    double part = 0.0, total;
    for (int s = threadIdx.x; s < segments; s += kThreads) part += lds.segment[s];
    (void)block_before(part, lds, total);
    return total;
}

// With the segments' sums in LDS: the first index whose running sum passes target(total); the last
// one with f > 0 where none does, -1 where there is none. Every thread gets it.
template <typename T>
struct Found {
    int at;
    T total;
};
template <typename T, int DT, typename F, typename G>
__device__ __forceinline__ Found<T> locate(const Row<DT>& row, Lds& lds, F f, G target_of)
{
    constexpr int N = Row<DT>::N;
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    const T* segment = segments_of(lds, T(0));
    if (threadIdx.x == 0) {
        lds.found_i[0] = kNone;
        lds.found_i[1] = -1;
    }
    __syncthreads();
    const int per = (row.segments + kThreads - 1) / kThreads;
    const int s0 = min((int)threadIdx.x * per, row.segments), s1 = min(s0 + per, row.segments);
    T mine = 0;
    for (int s = s0; s < s1; ++s) mine += segment[s];
    T total;
    const T before = block_before(mine, lds, total);
    const T target = target_of(total);
    // the first segment that passes the target, or the last one that has anything (the sums of
    // neighbouring threads may overlap or leave a gap by a rounding)
    T run = before, base = 0;
    int passed = kNone, last = -1;
    for (int s = s0; s < s1; ++s) {
        const T w = segment[s];
        if (w > 0) {
            if (passed == kNone && run + w > target) {
                passed = s;
                base = run;
            }
            last = s;
        }
        run += w;
    }
    const uint64_t hits = __ballot(passed != kNone), any = __ballot(last >= 0);
    if (hits && lane == __builtin_ctzll(hits)) atomicMin(&lds.found_i[0], passed);
    if (any && lane == 63 - __builtin_clzll(any)) atomicMax(&lds.found_i[1], last);
    __syncthreads();
    const int first = lds.found_i[0], s = first != kNone ? first : lds.found_i[1];
    if (first != kNone && passed == first) lds.found_d = (double)base;
    __syncthreads();
    base = (T)lds.found_d;
    if (s >= 0 && wave == 0) {
        const int chunk = s * kWave + lane;
        const Chunk<DT> c = row.at(chunk);
        T w[N], sum = 0;
        int top = -1;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            w[e] = f(c.x[e], chunk * N + e);
            sum += w[e];
            if (w[e] > 0) top = e;
        }
        T upto = base + (wave_scan(sum) - sum);
        int at = -1;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            upto += w[e];
            if (at < 0 && w[e] > 0 && upto > target) at = e;
        }
        const uint64_t hit = first != kNone ? __ballot(at >= 0) : 0, some = __ballot(top >= 0);
        const int winner = hit ? __builtin_ctzll(hit) : some ? 63 - __builtin_clzll(some) : 0;
        if (lane == winner) lds.found_i[2] = chunk * N + (hit ? at : top);
    }
    __syncthreads();
    const Found<T> out{s >= 0 ? lds.found_i[2] : -1, total};
    __syncthreads();
    return out;
}

template <typename T, int DT, typename F, typename G>
__device__ __forceinline__ Found<T> find_in_order(const Row<DT>& row, Lds& lds, F f, G target_of)
{
    sum_segments<T>(row, lds, f);
    return locate<T>(row, lds, f, target_of);
}

// Of kBins measures, two a thread from the top down, the first place (from the top) where their running
// sum from `base` on reaches the target, and what lies above it; `last_too`: of sums that end below it by a
// rounding, the last one that has anything. -1 where there is none.
struct Place {
    int at;
    double above;
};
__device__ __forceinline__ Place top_place(Lds& lds, double m0, double m1, double base, double target, bool last_too)
{
    const int lane = threadIdx.x & (kWave - 1);
    if (threadIdx.x == 0) {
        lds.found_i[0] = kBins;
        lds.found_i[1] = -1;
    }
    double total, run = base + block_before(m0 + m1, lds, total), above = 0.0;
    int place = kBins, last = -1;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const double m = q ? m1 : m0;
        if (m > 0.0) {
            last = 2 * (int)threadIdx.x + q;
            if (place == kBins && run + m >= target) {
                place = last;
                above = run;
            }
        }
        run += m;
    }
    const uint64_t hits = __ballot(place != kBins), any = __ballot(last >= 0);
    if (hits && lane == __builtin_ctzll(hits)) atomicMin(&lds.found_i[0], place);
    if (any && lane == 63 - __builtin_clzll(any)) atomicMax(&lds.found_i[1], last);
    __syncthreads();
    const int reached = lds.found_i[0], at = reached != kBins ? reached : last_too ? lds.found_i[1] : -1;
    const int mine = at - 2 * (int)threadIdx.x;
    if (at >= 0 && (mine == 0 || mine == 1)) lds.found_d = reached != kBins ? above : run - (mine == 0 ? m0 + m1 : m1);
    __syncthreads();
    const Place p{at, lds.found_d};
    __syncthreads();
    return p;
}

__device__ __forceinline__ void clear_bins(Lds& lds, bool masses)
{
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += kThreads) {
        if (masses) lds.mass[0][b] = lds.mass[1][b] = 0;
        else lds.count[b] = 0;
    }
    __syncthreads();
}

// The shares of a row and their largest logits; the first ones of each thread in registers.
struct Shares {
    static constexpr int kOwn = 4;
    const float* most;
    int n;
    float own[kOwn];
    __device__ __forceinline__ Shares(const float* most_, int n_) : most(most_), n(n_)
    {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int s = i * kThreads + (int)threadIdx.x;
            own[i] = s < n ? most[s] : -INFINITY;
        }
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const
    {
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
            if (i * kThreads + (int)threadIdx.x < n) f(i * kThreads + (int)threadIdx.x, own[i]);
        for (int s = kOwn * kThreads + (int)threadIdx.x; s < n; s += kThreads) f(s, most[s]);
    }
};

// A value that at least j of the shares' maxima reach and few more: the lower edge of a bin of those between `least`
// and the largest of them, `most`; -inf where there are fewer.
__device__ __forceinline__ float reached_by(Lds& lds, const Shares& shares, int j, float least, float most)
{
    const float scale = (float)(kBins - 1) / (most - least);
    if (!(scale > 0.0f) || !(scale < 3e38f)) return least < most ? -INFINITY : most;
    clear_bins(lds, false);
    shares.each([&](int, float x) {
        if (x >= least) atomicAdd(&lds.count[min((int)((x - least) * scale), kBins - 1)], 1u);
    });
    __syncthreads();
    const int b0 = kBins - 1 - 2 * (int)threadIdx.x;
    const Place p = top_place(lds, (double)lds.count[b0], (double)lds.count[b0 - 1], 0.0, (double)j, false);
    if (p.at < 0) return -INFINITY;
    // (a little below the edge, by what the bins' numbers round)
    const float edge = least + (float)(kBins - 1 - p.at) / scale;
    return edge - 4e-7f * (fabsf(edge) + fabsf(least) + fabsf(most));
}

// One token more in lds.packed, in no order: their ranks give them one.
__device__ __forceinline__ void push(Lds& lds, float x, int v)
{
    const int at = atomicAdd(&lds.n, 1);
    if (at < kList) lds.packed[at] = (uint64_t)key_of(x) << 32 | (uint32_t)~(uint32_t)v;
}

// The ones of `which` from index v on; few as a rule, and so read again.
template <int DT>
__device__ __forceinline__ void push_some(const Row<DT>& row, Lds& lds, uint32_t which, int v)
{
    for (; which; which &= which - 1) {
        const int i = v + __builtin_ctz(which);
        push(lds, row.value(i), i);
    }
}

// The tokens of `bound` and above in LDS: how many, which may be more than there is room for.
template <int DT>
__device__ __forceinline__ int collect(const Row<DT>& row, Lds& lds, const Shares& shares, int lanes, float bound)
{
    constexpr int N = Row<DT>::N;
    int some = 0, total;
    shares.each([&](int, float x) { some += x >= bound && x > -INFINITY ? 1 : 0; });
    int at = block_before(some, lds, total);
    if (total > kList) return total;
    if (threadIdx.x == 0) lds.n = 0;
    shares.each([&](int s, float x) {
        if (x >= bound && x > -INFINITY) lds.share[at++] = s;
    });
    __syncthreads();
    for (int j = (int)threadIdx.x / lanes; j < total; j += kThreads / lanes) {
        const int chunk = lds.share[j] * lanes + (int)threadIdx.x % lanes;
        const Chunk<DT> c = row.at(chunk);
        uint32_t which = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) which |= c.x[e] >= bound && c.x[e] > -INFINITY ? 1u << e : 0u;
        push_some(row, lds, which, chunk * N);
    }
    __syncthreads();
    const int n = lds.n;
    __syncthreads();
    return n;
}

// Every token of a row of at most kList.
template <int DT>
__device__ __forceinline__ int collect_all(const Row<DT>& row, Lds& lds)
{
    constexpr int N = Row<DT>::N;
    const Chunk<DT> c = row.at(threadIdx.x);
    uint32_t which = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) which |= c.x[e] > -INFINITY ? 1u << e : 0u;
    if (threadIdx.x == 0) lds.n = 0;
    __syncthreads();
    push_some(row, lds, which, (int)threadIdx.x * N);
    __syncthreads();
    const int n = lds.n;
    __syncthreads();
    return n;
}

// The values of threads 0 .. n-1 (above 0, all different; the others' count as 0) in descending order, one a thread. Few
// are compared each with each (50 tokens: a row 14.5 us, 19 by sorting; 430: 36, 34; 1,000: 45 more). More by a bitonic
// sort of as many as the next power of two: partners in a wavefront exchange by shuffles, others through LDS. All threads.
constexpr int kCompared = 256;
__device__ __forceinline__ uint64_t sorted(Lds& lds, uint64_t v, int n)
{
    const int t = threadIdx.x;
    if (n <= kCompared) {
        __syncthreads();
        if (t < n) lds.packed[t] = v;
        __syncthreads();
        int place = 0;
        if (uniform(t & ~(kWave - 1)) < n) {
#pragma unroll 4
            for (int j = 0; j < n; ++j) place += lds.packed[j] > v ? 1 : 0;
        }
        __syncthreads();
        if (t < n) lds.packed[place] = v;
        __syncthreads();
        return t < n ? lds.packed[t] : 0;
    }
    int size = 2;
    while (size < n) size <<= 1;
    if (t >= n) v = 0;
#pragma unroll 1
    for (int k = 2; k <= size; k <<= 1) {
#pragma unroll 1
        for (int j = k >> 1; j > 0; j >>= 1) {
            uint64_t o;
            if (j < kWave) o = __shfl_xor(v, j);
            else {
                __syncthreads();
                lds.packed[t] = v;
                __syncthreads();
                o = lds.packed[t ^ j];
            }
            // the upper part of a descending pair, the lower part of an ascending one, keeps the larger
            const bool larger = ((t & j) == 0) == ((t & k) == 0);
            v = (o > v) == larger ? o : v;
        }
    }
    return v;
}

// With n tokens in lds.packed, which are what comes in the order behind others of the weight `above`: which of
// them stay of a head of `most` tokens, or of the weight `target` (0: top_p of the n), with min_p. They are left in the
// list. False, and nothing changed but the order of lds.packed, where the head does not end among them. `light`: the head is `most`
// tokens, whatever top_p and min_p say.
__device__ __forceinline__ bool rank(Lds& lds, Dist& d, const Settings& set, int n, double most, double target, double above, bool light)
{
    const int t = threadIdx.x;
    uint64_t mine = t < n ? lds.packed[t] : 0;
    mine = sorted(lds, mine, n);
    // thread r has the token of rank r
    const float x = value_of((uint32_t)(mine >> 32));
    bool in = t < n && (double)t < most;
    const double w = in ? d.power(x) : 0.0;
    double sum;
    const double before = above + block_before(w, lds, sum);
    if (set.top_p < 1.0f && !light) {
        if (target > 0.0 && (above >= target || above + sum < target)) {
            __syncthreads();
            lds.packed[t] = mine;
            __syncthreads();
            return false;
        }
        const double of = target > 0.0 ? target : (double)set.top_p * sum;
        in = in && ((t == 0 && above == 0.0) || before < of);
    }
    if (set.min_p > 0.0f && !light) in = in && d.exponent(x) >= fmin(log2((double)set.min_p), 0.0);
    // (all of them a head of the order: their number says which)
    int kept;
    (void)block_before(in ? 1 : 0, lds, kept);
    (void)block_before(in ? w : 0.0, lds, d.total);
    if (t == kept - 1) {
        lds.found_d = (double)x;
        lds.found_i[0] = (int)~(uint32_t)mine;
    }
    // by index: the complements, which mine has in its lower half
    mine = sorted(lds, t < kept ? mine << 32 | __float_as_uint(x) : 0, kept);
    if (t < kept) {
        lds.list_x[t] = __uint_as_float((uint32_t)mine);
        lds.list_at[t] = (int)~(uint32_t)(mine >> 32);
    }
    __syncthreads();
    if (kept > 0) {
        d.cut = (float)lds.found_d;
        d.cut_at = lds.found_i[0];
    }
    d.kept = d.n = kept;
    __syncthreads();
    return true;
}

// With n tokens in lds.packed, among them all that stay in d: these into the list.
__device__ __forceinline__ void relist(Lds& lds, Dist& d, int n)
{
    const int t = threadIdx.x;
    uint64_t mine = t < n ? lds.packed[t] : 0;
    const float x = value_of((uint32_t)(mine >> 32));
    const bool in = t < n && d.stays(x, (int)~(uint32_t)mine);
    int kept;
    (void)block_before(in ? 1 : 0, lds, kept);
    mine = sorted(lds, in ? mine << 32 | __float_as_uint(x) : 0, n);  // (of what is 0 nothing is used)
    if (t < kept) {
        lds.list_x[t] = __uint_as_float((uint32_t)mine);
        lds.list_at[t] = (int)~(uint32_t)(mine >> 32);
    }
    d.n = kept;
    __syncthreads();
}

// A value's place among the ones between lo and hi of a type's keys: bf16 values differ in the upper half of theirs.
template <int DT>
struct Keys {
    static constexpr int kUnit = DT == kBF16 ? 16 : 0;
    __device__ static __forceinline__ uint32_t of(float x) { return key_of(x) >> kUnit; }
    // (of a bf16 value the lower half is zeros, of a negative one's key ones)
    __device__ static __forceinline__ float value(uint32_t k) { return value_of(kUnit && !(k & 0x8000u) ? k << kUnit | 0xFFFFu : k << kUnit); }
};

// A long head, of `k` tokens or of the weight `target` (0: by number) of `whole`, of the tokens that stay in d: with its end in d, the sums of
// its weights in lds.segment. False, and nothing changed, where the bins do not give its end. `lowest`: a logit that it
// does not go below.
template <int DT>
__device__ __forceinline__ bool long_head(const Row<DT>& row, Lds& lds, Dist& d, const Settings& set, float lowest, double k, double target, double whole)
{
    constexpr int N = Row<DT>::N;
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    const bool by_number = !(target > 0.0);
    const float m = (float)d.m, scale = (float)(kBins - 1) / (m - lowest), inv = (float)d.inv;
    if (!(scale > 0.0f) || !(scale < 3e38f)) return false;
    const bool all = !(d.cut > -INFINITY);  // every token of `lowest` and above stays in d
    // (rounded, but never out of the logits' order)
    auto bin_of = [&](float x) { return min((int)((x - lowest) * scale), kBins - 1); };
    // weights in units of which the whole has 2^31 (integers: an addition of floats in LDS takes some three clocks a
    // lane, and a flat row of 151,936 tokens 190 us)
    const float unit = by_number ? 0.0f : (float)(2147483648.0 / whole);
    const double each = by_number ? 1.0 : whole / 2147483648.0;
    clear_bins(lds, false);
    row.each([&](int, int v, const Chunk<DT>& c) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (c.x[e] >= lowest && (all || d.stays(c.x[e], v + e)))
                atomicAdd(&lds.count[bin_of(c.x[e])], by_number ? 1u : (uint32_t)fmaf(__builtin_amdgcn_exp2f((c.x[e] - m) * inv), unit, 0.5f));
    });
    __syncthreads();
    const int b0 = kBins - 1 - 2 * (int)threadIdx.x;
    const double m0 = (double)lds.count[b0] * each, m1 = (double)lds.count[b0 - 1] * each;
    // sums of 32-bit weights are off by less than one in 20,000 as a rule; what they give is checked below
    const double goal = by_number ? k : target;
    const Place from = top_place(lds, m0, m1, 0.0, by_number ? goal : goal * (1.0 - 5e-5), false);
    const Place to = by_number ? from : top_place(lds, m0, m1, 0.0, goal * (1.0 + 5e-5), true);
    if (from.at < 0 || to.at < 0) return false;
    const int upper = kBins - 1 - from.at, lower = kBins - 1 - to.at;
    // about how many tokens lie in these bins
    auto number_in = [&](int b, double mass) {
        return b > upper || b < lower || !(mass > 0.0) ? 0.0 : by_number ? mass : mass / fmax(d.power(fminf(lowest + ((float)b + 0.5f) / scale, m)), 1e-300);
    };
    double expected;
    (void)block_before(number_in(b0, m0) + number_in(b0 - 1, m1), lds, expected);
    // the least logits of the bins `lower` and `upper` + 1, by halves between two keys
    auto least_of = [&](int bin) {
        uint32_t a = key_of(lowest), z = key_of(m) + 1;  // (m lies in the last bin)
        while (a < z) {
            const uint32_t mid = a + (z - a) / 2;
            if (bin_of(value_of(mid)) >= bin) z = mid;
            else a = mid + 1;
        }
        return value_of(a);
    };
    const float x_lo = least_of(lower), x_hi = upper + 1 < kBins ? least_of(upper + 1) : INFINITY;
    // more of them than can be ranked are equal ones as a rule: counted by value then
    uint32_t* const values = (uint32_t*)lds.packed;
    const bool ranked = expected <= 0.95 * kList;
    uint32_t lo = 0;
    if (!ranked) {
        lo = Keys<DT>::of(x_lo);
        if (Keys<DT>::of(fminf(x_hi, m)) - lo >= (uint32_t)kBins) return false;
        static_assert(sizeof(uint64_t) * kList >= 4 * kBins, "");
        for (int b = threadIdx.x; b < kBins; b += kThreads) values[b] = 0;
    }
    if (threadIdx.x == 0) lds.n = 0;
    __syncthreads();
    int over = 0;
    row.template each<2>([&](int i, int v, const Chunk<DT>& c) {
        double s = 0.0;
        uint32_t which = 0;
#pragma unroll
        for (int h = 0; h < N; h += 4) {
            double w[4];
            uint32_t in = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = c.x[h + e];
                const bool some = x >= x_lo && (all || d.stays(x, v + h + e));
                in |= some && x >= x_hi ? 1u << e : 0u;
                which |= some && x < x_hi ? 1u << (h + e) : 0u;
                w[e] = (double)x - d.m;
            }
            over += __popc(in);
            if (in) {
                exp2_of(d.table, w, d.inv, d.zero);
#pragma unroll
                for (int e = 0; e < 4; ++e) s += in >> e & 1 ? w[e] : 0.0;
            }
        }
        if (ranked) push_some(row, lds, which, v);
        else
            for (; which; which &= which - 1) {
                const uint32_t at = Keys<DT>::of(row.value(v + __builtin_ctz(which))) - lo;
                if (at < (uint32_t)kBins) atomicAdd(&values[at], 1u);
            }
        s = wave_scan(s);
        if (lane == kWave - 1) lds.segment[i * kWaves + wave] = s;
    });
    __syncthreads();
    const int n = lds.n;
    const double above = sum_of_segments(lds, row.segments);
    int number;
    (void)block_before(over, lds, number);
    Dist next = d;
    next.summed = true;
    next.listed = false;
    if (!ranked) {
        if (by_number ? (double)number >= k : above >= target) return false;
        auto measure = [&](int b) { return by_number || values[b] == 0 ? (double)values[b] : (double)values[b] * d.power(Keys<DT>::value(lo + (uint32_t)b)); };
        const Place p = top_place(lds, measure(b0), measure(b0 - 1), by_number ? (double)number : above, goal, false);
        if (p.at < 0) return false;
        const int bin = kBins - 1 - p.at;
        const double w = by_number ? 1.0 : d.power(Keys<DT>::value(lo + (uint32_t)bin)), there = (double)values[bin];
        double some = fmax(ceil((goal - p.above) / w), 1.0);
        if (some > 1.0 && p.above + (some - 1.0) * w >= goal) some -= 1.0;
        some = fmin(some, there);
        const float x0 = Keys<DT>::value(lo + (uint32_t)bin);
        next.cut_at = x0 == d.cut ? d.cut_at : kNone;  // (all that stay: of the value that d ends in, those that d has)
        next.cut = x0;
        if (some < there) {
            next.cut_at = find_in_order<int>(row, lds, [&](float x, int v) { return x == x0 && d.stays(x, v) ? 1 : 0; }, [&](int) { return (int)some - 1; }).at;
        }
        // the weights of these bins' tokens that stay join their segments
        int inside = 0;
        row.template each<2>([&](int i, int v, const Chunk<DT>& c) {
            double s = 0.0;
            bool any = false;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float x = c.x[e];
                if (x >= x_lo && x < x_hi && next.stays(x, v + e)) {
                    s += d.power(x);
                    any = true;
                    ++inside;
                }
            }
            if (!__ballot(any)) return;
            s = wave_scan(s);
            if (lane == kWave - 1) lds.segment[i * kWaves + wave] += s;
        });
        __syncthreads();
        (void)block_before(inside, lds, next.kept);
        next.kept += number;
        next.total = sum_of_segments(lds, row.segments);
        d = next;
        return true;
    }
    if (n < 1 || n > kList) return false;
    if (by_number) {
        if ((double)number >= k || (double)(number + n) < k) return false;
        (void)rank(lds, next, set, n, k - (double)number, 0.0, above, true);
    } else {
        Settings p = set;
        p.min_p = 0.0f;
        if (!rank(lds, next, p, n, (double)n, target, above, false)) return false;
    }
    // the tokens of these bins that stay join their segments, each segment's in the order of their indices
    const int stay = next.n;
    if ((int)threadIdx.x < stay) {
        const int t = threadIdx.x;
        auto segment = [&](int i) { return lds.list_at[i] / (kWave * N); };
        const int mine = segment(t);
        if (t == 0 || segment(t - 1) != mine) {
            double s = lds.segment[mine];
            for (int i = t; i < stay && segment(i) == mine; ++i) s += d.power(lds.list_x[i]);
            lds.segment[mine] = s;
        }
    }
    __syncthreads();
    next.kept += number;
    next.total += above;
    d = next;
    return true;
}

// Where the order of the tokens that stay in d reaches the target: the key's value, how many tokens of that
// value belong to the head, and whether these are all. Counted, or weighed.
struct Cut {
    bool there, all;
    float x;
    double n;
};
// (a weight is at most 1 and a row has at most 2^20: 2^43 of them stay below 2^63)
template <bool MASS, int DT>
__device__ __forceinline__ Cut cut_of(const Row<DT>& row, Lds& lds, const Dist& d, float lowest, double target)
{
    constexpr int N = Row<DT>::N;
    constexpr double kHi = 8796093022208.0, kInvHi = 1.0 / kHi;  // 2^43
    uint32_t lo = Keys<DT>::of(lowest), hi = Keys<DT>::of((float)d.m);
    double above = 0.0;
    bool first = true;
#pragma unroll 1
    while (true) {
        int shift = 0;
        while ((hi - lo) >> shift >= (uint32_t)kBins) ++shift;
        const bool exact = shift == 0;  // a bin is a value: counting weighs it
        clear_bins(lds, MASS && !exact);
        row.template each<2>([&](int, int v, const Chunk<DT>& c) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t k = Keys<DT>::of(c.x[e]);
                if (k < lo || k > hi || !d.stays(c.x[e], v + e)) continue;
                const int bin = (int)((k - lo) >> shift);
                if (MASS && !exact) {
                    const double w = d.power(c.x[e]) * kHi;
                    const uint64_t up = (uint64_t)w;
                    atomicAdd((unsigned long long*)&lds.mass[0][bin], up);
                    atomicAdd((unsigned long long*)&lds.mass[1][bin], (uint64_t)((w - (double)up) * kHi));
                } else atomicAdd(&lds.count[bin], 1u);
            }
        });
        __syncthreads();
        auto value = [&](uint32_t k) { return Keys<DT>::value(k); };
        auto measure = [&](int bin) {
            if (!MASS) return (double)lds.count[bin];
            if (!exact) return (double)lds.mass[0][bin] * kInvHi + (double)lds.mass[1][bin] * (kInvHi * kInvHi);
            const uint32_t n = lds.count[bin];
            return n ? (double)n * d.power(value(lo + (uint32_t)bin)) : 0.0;
        };
        const int b0 = kBins - 1 - 2 * (int)threadIdx.x;
        const Place p = top_place(lds, measure(b0), measure(b0 - 1), above, target, !first);
        if (p.at < 0) return Cut{false, false, 0.0f, 0.0};
        first = false;
        above = p.above;
        const uint32_t bin = (uint32_t)(kBins - 1 - p.at);
        if (exact) {
            Cut cut;
            cut.there = true;
            cut.x = value(lo + bin);
            const double w = MASS ? d.power(cut.x) : 1.0, count = (double)lds.count[bin];
            double n = fmax(ceil((target - above) / w), 1.0);
            if (n > 1.0 && above + (n - 1.0) * w >= target) n -= 1.0;
            cut.n = fmin(n, count);
            cut.all = cut.n == count;
            __syncthreads();
            return cut;
        }
        lo += bin << shift;
        hi = min(hi, lo + ((1u << shift) - 1));
    }
}

// The segments' sums that the scan left, relative to the row's largest logit.
template <int DT>
__device__ __forceinline__ void spread_sums(const Row<DT>& row, Lds& lds, const RowScan& scan, const Dist& d)
{
    __syncthreads();
    for (int s = threadIdx.x; s < row.segments; s += kThreads) {
        const float of = scan.of[s];
        lds.segment[s] = of > -INFINITY ? scan.sum[s] * d.power(of) : 0.0;
    }
    __syncthreads();
}

// One segment's sum of f(x, v).
template <int DT, typename F>
__device__ __forceinline__ void sum_again(const Row<DT>& row, Lds& lds, int segment, F f)
{
    constexpr int N = Row<DT>::N;
    const int lane = threadIdx.x & (kWave - 1);
    if ((int)threadIdx.x < kWave) {
        const int chunk = segment * kWave + lane;
        const Chunk<DT> c = row.at(chunk);
        double s = 0.0;
#pragma unroll
        for (int e = 0; e < N; ++e) s += f(c.x[e], chunk * N + e);
        s = wave_scan(s);
        if (lane == kWave - 1) lds.segment[segment] = s;
    }
    __syncthreads();
}

// The segments' sums of the weights, the whole and the number, of a distribution that has none of them.
template <int DT>
__device__ __forceinline__ void weigh_again(const Row<DT>& row, Lds& lds, Dist& d)
{
    int stay = 0;
    sum_segments<double>(row, lds, [&](float x, int v) {
        if (!d.stays(x, v)) return 0.0;
        ++stay;
        return d.power(x);
    });
    d.total = sum_of_segments(lds, row.segments);
    (void)block_before(stay, lds, d.kept);
    d.summed = true;
}

template <int DT>
__device__ __forceinline__ Dist solve(const Row<DT>& row, Lds& lds, const Settings& set, const RowScan& scan, int lanes)
{
    constexpr int N = Row<DT>::N;
    constexpr float kLowest = -3.402823466e38f;
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    Dist d;
    d.table = lds.s.table;
    d.inv = inverse_of(set.temperature);
    d.zero = kLeast / d.inv;
    d.cut = -INFINITY;
    d.cut_at = -1;
    d.least = -INFINITY;
    d.listed = d.summed = false;
    d.best = d.kept = -1;
    d.n = 0;
    d.total = 0.0;
    const bool small = row.vocab <= kList;  // every token is ranked: no scan
    const int n_shares = small ? 0 : row.segments * (kWave / lanes);
    const Shares shares(scan.most, n_shares);
    float mine = -INFINITY, low = INFINITY;
    bool bad = false;
    auto look = [&](float x) {
        bad = bad || !(x < INFINITY);
        mine = fmaxf(mine, x);
        low = x > -INFINITY ? fminf(low, x) : low;
    };
    if (small) {
        const Chunk<DT> c = row.at(threadIdx.x);
#pragma unroll
        for (int e = 0; e < N; ++e) look(c.x[e]);
    } else
        shares.each([&](int, float x) { look(x); });
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
        mine = fmaxf(mine, __shfl_xor(mine, s));
        low = fminf(low, __shfl_xor(low, s));
    }
    const bool wave_bad = __ballot(bad) != 0;
    int* room = lds.room(0);
    if (lane == 0) {
        lds.s.wave_f[0][wave] = mine;
        lds.s.wave_f[1][wave] = low;
        room[wave] = wave_bad;
    }
    if (threadIdx.x == 0) {
        lds.found_i[0] = kNone;
        lds.n = 0;
    }
    __syncthreads();
    float m = mine;
    bool any_bad = false;
#pragma unroll 4
    for (int w = 0; w < kWaves; ++w) {
        m = fmaxf(m, lds.s.wave_f[0][w]);
        low = fminf(low, lds.s.wave_f[1][w]);
        any_bad = any_bad || room[w] != 0;
    }
    __syncthreads();
    d.none = any_bad || m == -INFINITY;
    d.m = m;
    if (d.none) return d;
    if (set.greedy()) {  // the largest alone: the first of equal ones
        int s = kNone;
        if (small) s = threadIdx.x;
        else {
            shares.each([&](int i, float x) { s = x == m ? min(s, i) : s; });
            if (s != kNone) atomicMin(&lds.found_i[0], s);
            __syncthreads();
            s = lds.found_i[0] * lanes + (int)threadIdx.x;
            __syncthreads();
            if (threadIdx.x == 0) lds.found_i[0] = kNone;
            __syncthreads();
        }
        const Chunk<DT> c = row.at(s);
        int at = kNone;
#pragma unroll
        for (int e = N - 1; e >= 0; --e) at = c.x[e] == m ? s * N + e : at;
        if (at != kNone && (small || (int)threadIdx.x < lanes)) atomicMin(&lds.found_i[0], at);
        __syncthreads();
        d.best = d.cut_at = lds.found_i[0];
        d.inv = 0.0;
        d.zero = -1.0;
        d.cut = m;
        d.kept = 1;
        d.total = 1.0;
        __syncthreads();
        return d;
    }

    const bool by_k = set.by_k(row.vocab), sums = !small && set.sums(row.vocab);
    const int k = by_k ? set.top_k : row.vocab;
    double whole = 0.0;
    if (sums) {
        spread_sums(row, lds, scan, d);
        whole = sum_of_segments(lds, row.segments);
        if (!(set.top_p < 1.0f)) {
            d.summed = true;
            d.total = whole;
            return d;
        }
    }
    // a short head: its tokens, or more than there is room for
    const double target = (double)set.top_p * whole;
    // (of the shares' maxima, those that 2^-100 of the largest weight and more belong to)
    const float floor = fmaxf(low, fmaxf((float)(d.m - 100.0 / d.inv), kLowest));
    // below it min_p leaves nothing (and, by the rounding of the bound, above it some)
    auto lightest = [&] {
        const float b = (float)(d.m + (log2(fmin((double)set.min_p, 1.0)) - 1e-3) / d.inv);
        return b - fabsf(b) * 1e-6f;
    };
    float bound = -INFINITY;
    int n = 0;
    bool all_of_min_p = false;  // the tokens listed are all that min_p leaves
    if (small) {
        n = collect_all(row, lds);
    } else {
        bool attempt = true;
        if (by_k) {
            attempt = k <= kList;
            if (attempt) bound = reached_by(lds, shares, k, floor, m);
        } else if (sums) {
            attempt = target < (double)kList;  // (no weight is above 1)
            if (attempt) bound = reached_by(lds, shares, kTryHead, floor, m);
            if (set.min_p > 0.0f && (!attempt || lightest() >= bound)) {
                bound = lightest();
                attempt = all_of_min_p = true;
            }
        } else bound = lightest();  // min_p alone
        if (attempt) n = collect(row, lds, shares, lanes, bound);
    }
    const bool enough = !by_k || n >= k || !(bound > -INFINITY);  // (or all there are)
    if (enough && n > 0 && n <= kList && rank(lds, d, set, n, (double)min(k, n), sums ? fmax(target, 1e-300) : 0.0, 0.0, false)) {
        d.listed = true;
        return d;
    }
    __syncthreads();
    if (!small && sums && set.min_p > 0.0f) {  // what min_p leaves: top_p's head ends in it, or it is all that stays
        if (!all_of_min_p) n = collect(row, lds, shares, lanes, lightest());
        if (n > 0 && n <= kList) {
            Settings alone = set;
            alone.top_p = 1.0f;
            if (all_of_min_p || !rank(lds, d, set, n, (double)n, fmax(target, 1e-300), 0.0, false)) (void)rank(lds, d, alone, n, (double)n, 0.0, 0.0, false);
            d.listed = true;
            return d;
        }
        __syncthreads();
    }

    // a long one
    auto narrow = [&](const Cut& c) {
        const Dist before = d;
        d.kept = -1;
        d.summed = false;
        d.cut_at = c.x == before.cut ? before.cut_at : kNone;  // (all that stay of that value)
        if (!c.all)  // the first of them
            d.cut_at = find_in_order<int>(row, lds, [&](float x, int v) { return x == c.x && before.stays(x, v) ? 1 : 0; },
                                          [&](int) { return (int)c.n - 1; }).at;
        d.cut = c.x;
    };
    if (by_k) {
        // (a head of more tokens than are ranked: about the logit that it ends above. Most shares of 16 loads have
        // a few above the least of their maxima; below 2^-60 of the largest weight there is little to end it)
        float near = bound;
        if (k > kList && k <= 2 * n_shares) near = floor;
        if (!(near > -INFINITY)) near = fmaxf((float)(d.m - 60.0 / d.inv), kLowest);
        if (!long_head(row, lds, d, set, near, (double)k, 0.0, 0.0)) {
            const Cut c = cut_of<false>(row, lds, d, kLowest, (double)k);
            if (c.there) narrow(c);
        }
    }
    if (set.top_p < 1.0f && !sums) {
        if (d.kept < 0) weigh_again(row, lds, d);
        whole = d.total;
    }
    const double goal = fmax((double)set.top_p * whole, 1e-300);
    if (set.min_p > 0.0f) {  // what it leaves is all that stays, if that weighs less than top_p's head: else it leaves that head
        Dist t = d;
        t.least = fmin(log2((double)set.min_p), 0.0);
        if (lightest() > t.cut) {  // (so that these can be listed without reading the row)
            t.cut = lightest();
            t.cut_at = kNone;
        }
        weigh_again(row, lds, t);
        if (!(set.top_p < 1.0f) || t.total < goal) return t;
        d.summed = false;
    }
    if (set.top_p < 1.0f) {
        // the tokens below a (1 - top_p) / vocab of the whole are less than (1 - top_p) of it together; at
        // least the first stays
        const double share = fmax((1.0 - (double)set.top_p) * whole / (double)row.vocab, 1e-300);
        const double low = d.m + (log2(fmin(share, 1.0)) - 1e-3) / d.inv;
        const float lowest = fmaxf((float)(low - fabs(low) * 1e-6), kLowest);
        if (!long_head(row, lds, d, set, lowest, 0.0, goal, whole)) {
            const Cut c = cut_of<true>(row, lds, d, lowest, goal);
            if (c.there) narrow(c);
        }
    }
    return d;
}

// u as the running sum's target: [0, 1), NaN as 0.
__device__ __forceinline__ double drawn(float u, double total) { return (u > 0.0f ? (double)u : 0.0) * total; }

// Of the list, the first token whose running sum of f(x, v) >= 0 passes u times the whole; -1 where nothing is.
template <typename F>
__device__ __forceinline__ Found<double> pick_listed(Lds& lds, const Dist& d, float u, F f)
{
    const int t = threadIdx.x, lane = t & (kWave - 1);
    const double w = t < d.n ? f(lds.list_x[t], lds.list_at[t]) : 0.0;
    if (t == 0) {
        lds.found_i[0] = kNone;
        lds.found_i[1] = -1;
    }
    double total;
    const double before = block_before(w, lds, total), target = drawn(u, total);
    const uint64_t hits = __ballot(w > 0.0 && before + w > target), any = __ballot(w > 0.0);
    if (hits && lane == __builtin_ctzll(hits)) atomicMin(&lds.found_i[0], t);
    if (any && lane == 63 - __builtin_clzll(any)) atomicMax(&lds.found_i[1], t);
    __syncthreads();
    const int s = lds.found_i[0] != kNone ? lds.found_i[0] : lds.found_i[1];
    const Found<double> out{s >= 0 ? lds.list_at[s] : -1, total};
    __syncthreads();
    return out;
}

// A token of a distribution that is listed, summed or one token.
template <int DT>
__device__ __forceinline__ int draw(const Row<DT>& row, Lds& lds, const Dist& d, float u)
{
    if (d.best >= 0) return d.best;
    auto weight = [&](float x, int v) { return d.weight(x, v); };
    if (d.listed) return pick_listed(lds, d, u, weight).at;
    return locate<double>(row, lds, weight, [&](double total) { return drawn(u, total); }).at;
}

// ln p of token v.
template <int DT>
__device__ __forceinline__ float logprob_of(const Row<DT>& row, const Dist& d, int v)
{
    return (float)((d.exponent(row.value(v)) - log2(d.total)) * kLn2);
}

template <int DT>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a)
{
    __shared__ Scratch scratch;
    Lds lds(scratch);
    fill_table(scratch.table);
    const int r = a.first + (int)blockIdx.x;
    const Row<DT> row(a.logits, r, a.vocab);
    Dist d = solve(row, lds, settings_of(a.set, r), scan_of(a.scan, r), a.scan.lanes);
    int token = -1, kept = 0;
    if (!d.none) {
        if (d.kept < 0 && !d.summed) weigh_again(row, lds, d);
        token = draw(row, lds, d, a.u[r]);
        kept = d.kept;
        if (a.kept && kept < 0) {  // (every one above -inf)
            const RowScan scan = scan_of(a.scan, r);
            int n = 0;
            for (int s = threadIdx.x; s < row.segments; s += kThreads) n += scan.number[s];
            (void)block_before(n, lds, kept);
        }
    }
    if (threadIdx.x != 0) return;
    if (a.token) a.token[r] = token;
    if (a.kept) a.kept[r] = kept;
    if (a.logprob) a.logprob[r] = token < 0 ? __builtin_nanf("") : logprob_of(row, d, token);
}

// The distributions of a verification, the rows' and the drafts' ones side by side: of each what weighs a token.
template <int DT>
__global__ __launch_bounds__(kThreads) void k_distribute(VerifyArgs a)
{
    __shared__ Scratch scratch;
    Lds lds(scratch);
    fill_table(scratch.table);
    const int block = a.first + (int)blockIdx.x, pairs = a.n_seqs * a.ch.max_new, which = block >= pairs ? 1 : 0;
    const int s = (block - which * pairs) / a.ch.max_new, i = block - which * pairs - s * a.ch.max_new;
    const Rows rows = seq_rows(a.ch, s);
    if (i >= min(rows.n, a.ch.max_new) - which) return;
    const int r = rows.begin + i;
    const int64_t at = dist_at(a.ch, which, r);
    const Row<DT> row(which ? a.draft : a.logits, r, a.vocab);
    Dist d = solve(row, lds, settings_of(a.set, r), scan_of(a.scan, at), a.scan.lanes);
    if (!d.none && d.kept < 0 && !d.summed) weigh_again(row, lds, d);
    if (threadIdx.x == 0) a.known[at] = Known{d.m, d.inv, d.zero, d.least, d.total, d.cut, d.cut_at, d.kept, d.best, d.none ? 1 : 0};
}

__device__ __forceinline__ Dist known_of(const Known& k, const double* table)
{
    Dist d;
    d.none = k.none != 0;
    d.listed = d.summed = false;
    d.best = k.best;
    d.kept = k.kept;
    d.n = 0;
    d.m = k.m;
    d.inv = k.inv;
    d.zero = k.zero;
    d.cut = k.cut;
    d.cut_at = k.cut_at;
    d.least = k.least;
    d.total = k.total;
    d.table = table;
    return d;
}

// What is asked of row r of a sequence: whether the draft behind it stands, and of what its token is drawn where it does not.
struct Answer {
    Dist p, q;
    double qt;          // q's whole
    int draft;          // -1 behind the last row
    bool last, certain; // the draft was drawn from no distribution
    bool yes;
    // what p has more than q, of the last row p itself
    __device__ __forceinline__ double more(double w, double z, int v) const
    {
        if (last || certain) return v == draft ? 0.0 : w;
        const double has = w * qt, over = has - z * p.total;
        return over > has * kSame ? over : 0.0;
    }
    __device__ __forceinline__ bool alone() const { return last || certain; }
    // whether so many tokens may be drawn that the row's segments are summed by k_verify_sums
    __device__ __forceinline__ bool many() const
    {
        return !p.none && !yes && p.best < 0 && (p.kept < 0 ? !alone() : p.kept > kList);
    }
};
template <int DT>
__device__ __forceinline__ Answer answer_of(const VerifyArgs& a, const double* table, const Row<DT>& row, const Row<DT>& other, int r, bool last, bool has_draft)
{
    Answer w;
    w.p = known_of(a.known[r], table);
    w.q = known_of(a.known[dist_at(a.ch, has_draft ? 1 : 0, r)], table);
    w.last = last;
    w.certain = !has_draft || w.q.none;
    w.qt = w.certain ? 1.0 : w.q.total;
    w.draft = last ? -1 : a.tokens[r + 1];
    w.yes = false;
    if (!w.p.none && w.draft >= 0 && w.draft < a.vocab) {
        const double ua = a.u_accept[r] > 0.0f ? (double)a.u_accept[r] : 0.0;
        const double qd = w.certain ? 1.0 : w.q.weight(other.value(w.draft), w.draft);
        w.yes = ua * qd * w.p.total < w.p.weight(row.value(w.draft), w.draft) * w.qt;
    }
    return w;
}
// (a row of which more than kList tokens stay, or of which all do and the draft was drawn)
__device__ __forceinline__ bool may_be_many(const VerifyArgs& a)
{
    return a.scan.parts > 0 && (a.draft.base || a.set.top_k || a.set.top_p || a.set.min_p);
}

// The segments' sums of what the token of a row is drawn from, where many may be: by many workgroups a row, as few rows
// have them: 256 rows of 151,936 bf16 logits and their drafts' 20 us (by each row's own one 72-100 with k_verify's 16; by as many
// workgroups as read the rows first 44). Bound by the 64-bit weights of both rows.
constexpr int64_t kSumsTarget = 8192;
template <int DT>
__global__ __launch_bounds__(kScanThreads) void k_verify_sums(VerifyArgs a, int parts, int per)
{
    constexpr int N = Chunk<DT>::N, kAhead = 2;
    __shared__ double table[kTable];
    fill_table(table);
    const int item = blockIdx.x / parts, part = blockIdx.x - item * parts;
    const int s = item / a.ch.max_new, i = item - s * a.ch.max_new;
    const Rows rows = seq_rows(a.ch, s);
    const int n = min(rows.n, a.ch.max_new);
    if (i >= n) return;
    const int r = rows.begin + i, lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    const bool last = i == n - 1, has_draft = a.draft.base && !last;
    const Row<DT> row(a.logits, r, a.vocab), other(has_draft ? a.draft : a.logits, r, a.vocab);
    const Answer w = answer_of(a, table, row, other, r, last, has_draft);
    if (!w.many()) return;
    const RowScan scan = scan_of(a.scan, r);
    const int first = part * per, end = min(first + per, row.segments);
#pragma unroll 1
    for (int s0 = first + wave; s0 < end; s0 += kScanWaves * kAhead) {
        u32x4 mine[kAhead], its[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int chunk = min(s0 + e * kScanWaves, end - 1) * kWave + lane;
            mine[e] = row.load(chunk);
            its[e] = w.alone() ? mine[e] : other.load(chunk);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int at = s0 + k * kScanWaves, v = (at * kWave + lane) * N;
            if (at >= end) break;
            Chunk<DT> x(mine[k]), y(its[k]);
            x.end(a.vocab - v);
            y.end(a.vocab - v);
            double sum = 0.0;
#pragma unroll
            for (int h = 0; h < N; h += 4) {
                double by[4], to[4], z[4];
                uint32_t in = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    by[e] = (double)x.x[h + e] - w.p.m;
                    to[e] = (double)y.x[h + e] - w.q.m;
                    in |= w.p.stays(x.x[h + e], v + h + e) && by[e] >= w.p.zero ? 1u << e : 0u;
                    z[e] = 0.0;
                }
                if (!in) continue;
                exp2_of(table, by, w.p.inv, w.p.zero);
                if (!w.alone()) {
                    uint32_t q = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) q |= w.q.stays(y.x[h + e], v + h + e) && to[e] >= w.q.zero ? 1u << e : 0u;
                    exp2_of(table, to, w.q.inv, w.q.zero);
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[e] = q >> e & 1 ? to[e] : 0.0;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += in >> e & 1 ? w.more(by[e], z[e], v + h + e) : 0.0;
            }
            sum = wave_scan(sum);
            if (lane == kWave - 1) scan.sum[at] = sum;
        }
    }
}

// Row i of sequence s: whether its draft stands, and the token that follows it.
template <int DT>
__global__ __launch_bounds__(kThreads) void k_verify(VerifyArgs a)
{
    __shared__ Scratch scratch;
    Lds lds(scratch);
    fill_table(scratch.table);
    const int block = a.first + (int)blockIdx.x, s = block / a.ch.max_new, i = block - s * a.ch.max_new;
    const Rows rows = seq_rows(a.ch, s);
    const int n = min(rows.n, a.ch.max_new);
    if (i >= n) return;
    const int r = rows.begin + i;
    const bool last = i == n - 1, has_draft = a.draft.base && !last;
    const Row<DT> row(a.logits, r, a.vocab), other(has_draft ? a.draft : a.logits, r, a.vocab);
    Answer w = answer_of(a, scratch.table, row, other, r, last, has_draft);
    Dist& p = w.p;
    int token = -1;
    if (!p.none) {
        if (w.yes) token = w.draft;
        else {
            const float u = a.u[r];
            auto more = [&](float x, float y, int v) {
                const double mine = p.weight(x, v);
                return w.alone() || mine > 0.0 ? w.more(mine, w.alone() ? 0.0 : w.q.weight(y, v), v) : 0.0;
            };
            auto one = [&](float x, int v) { return more(x, w.alone() ? 0.0f : other.value(v), v); };
            auto weight = [&](float x, int v) { return p.weight(x, v); };
            // few tokens are listed again; of more the row's sums are there, or it is read
            bool listed = false;
            if (p.kept > 0 && p.kept <= kList && p.best < 0) {
                int m;
                if (a.vocab <= kList) m = collect_all(row, lds);
                else {
                    const RowScan scan = scan_of(a.scan, r);
                    m = collect(row, lds, Shares(scan.most, a.scan.shares), a.scan.lanes, p.cut);
                }
                listed = m > 0 && m <= kList;
                if (listed) relist(lds, p, m);
            }
            if (p.best >= 0) token = p.best == w.draft ? -1 : p.best;
            else if (listed) token = pick_listed(lds, p, u, one).at;
            else {
                if (w.many() && may_be_many(a)) {
                    const RowScan scan = scan_of(a.scan, r);
                    for (int at = threadIdx.x; at < row.segments; at += kThreads) lds.segment[at] = scan.sum[at];
                    __syncthreads();
                } else if (p.kept < 0 && w.alone()) {  // every token stays: the segments' sums are known, but for the draft's
                    spread_sums(row, lds, scan_of(a.scan, r), p);
                    if (w.draft >= 0 && w.draft < a.vocab) sum_again(row, lds, w.draft / (kWave * Row<DT>::N), one);
                } else sum_segments<double>(row, lds, other, more);
                token = locate<double>(row, lds, one, [&](double t) { return drawn(u, t); }).at;
            }
            if (token < 0) {  // (nothing more)
                if (p.best >= 0) token = p.best;
                else if (listed) token = pick_listed(lds, p, u, weight).at;
                else token = find_in_order<double>(row, lds, weight, [&](double t) { return drawn(u, t); }).at;
            }
        }
    }
    if (threadIdx.x != 0) return;
    a.row_token[r] = token;
    a.row_yes[r] = w.yes ? 1 : 0;
    a.row_logprob[r] = token < 0 ? __builtin_nanf("") : logprob_of(row, p, token);
}

// A sequence's drafts stand up to the first that does not; a wavefront a sequence.
__global__ __launch_bounds__(256) void k_verify_join(VerifyArgs a)
{
    const int s = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & (kWave - 1);
    if (s >= a.n_seqs) return;
    const Rows rows = seq_rows(a.ch, s);
    const int n = min(rows.n, a.ch.max_new);
    int stop = n;
    for (int i0 = 0; i0 < n && stop == n; i0 += kWave) {
        const uint64_t no = __ballot(i0 + lane < n && a.row_yes[rows.begin + min(i0 + lane, n - 1)] == 0);
        if (no) stop = i0 + __builtin_ctzll(no);
    }
    for (int i = lane; i < n; i += kWave) {
        const int r = rows.begin + i;
        if (a.next) a.next[r] = i <= stop ? a.row_token[r] : -1;
        if (a.logprob) a.logprob[r] = i <= stop ? a.row_logprob[r] : __builtin_nanf("");
    }
    if (lane != 0) return;
    const int accepted = n > 0 ? stop : 0;
    if (a.accepted) a.accepted[s] = accepted;
    if (a.length_out) a.length_out[s] = a.length[s] - (n > 0 ? rows.n - 1 - accepted : 0);
}

template <typename K, typename... A>
int enqueue(K kernel, int64_t blocks, int threads, void* stream, void* ev0, void* ev1, const A&... a)
{
    if (blocks <= 0) return kNoLaunch;
    if (ev0 && ev1)
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, (hipStream_t)stream, (hipEvent_t)ev0, (hipEvent_t)ev1, 0, a...);
    else
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, (hipStream_t)stream, a...);
    return (int)hipGetLastError();
}

}  // namespace

// Shares of a row by the loads of 16 bytes that it has: 1,024 or more of them where there are as many loads, and not
// many more, so that their maxima take little beside the row.
void scan_shape(ScanDev& d, int64_t rows, int64_t vocab, int dtype)
{
    const int64_t per_load = dtype == kBF16 ? 8 : 4, chunks = (vocab + per_load - 1) / per_load, segments = (chunks + kWave - 1) / kWave;
    d.lanes = chunks <= 2048 ? 1 : chunks <= 8192 ? 4 : 16;
    d.segments = (int32_t)segments;
    d.shares = (int32_t)(segments * (kWave / d.lanes));
    // workgroups of one segment a wavefront at least, and about kScanTarget of them
    const int64_t each = (rows * segments + kScanTarget * kScanWaves - 1) / (kScanTarget * kScanWaves);
    d.per = (int32_t)(std::max<int64_t>(1, std::min(each, (segments + kScanWaves - 1) / kScanWaves)) * kScanWaves);
    d.parts = (int32_t)((segments + d.per - 1) / d.per);
    if (vocab <= kList) d.parts = d.segments = d.shares = 0;
}

namespace {

template <int DT>
int scan_rows(const SampleArgs& a, void* st, void* e0, void* e1)
{
    const int64_t blocks = (int64_t)a.rows * a.scan.parts;
    return a.scan.lanes == 1   ? enqueue(k_scan<DT, 1>, blocks, kScanThreads, st, e0, e1, a)
           : a.scan.lanes == 4 ? enqueue(k_scan<DT, 4>, blocks, kScanThreads, st, e0, e1, a)
                               : enqueue(k_scan<DT, 16>, blocks, kScanThreads, st, e0, e1, a);
}

template <int DT>
int verify_scan_rows(const VerifyArgs& a, void* st, void* e0, void* e1)
{
    return a.scan.lanes == 1   ? enqueue(k_verify_scan<DT, 1>, a.blocks, kScanThreads, st, e0, e1, a)
           : a.scan.lanes == 4 ? enqueue(k_verify_scan<DT, 4>, a.blocks, kScanThreads, st, e0, e1, a)
                               : enqueue(k_verify_scan<DT, 16>, a.blocks, kScanThreads, st, e0, e1, a);
}

}  // namespace

int launch_scan(const SampleArgs& a, void* st, void* e0, void* e1)
{
    return a.dtype == kBF16 ? scan_rows<kBF16>(a, st, e0, e1) : scan_rows<kF32>(a, st, e0, e1);
}

int launch_verify_scan(const VerifyArgs& a, void* st, void* e0, void* e1)
{
    return a.dtype == kBF16 ? verify_scan_rows<kBF16>(a, st, e0, e1) : verify_scan_rows<kF32>(a, st, e0, e1);
}

int launch_sample(const SampleArgs& a, void* st, void* e0, void* e1)
{
    return a.dtype == kBF16 ? enqueue(k_sample<kBF16>, a.blocks, kThreads, st, e0, e1, a)
                            : enqueue(k_sample<kF32>, a.blocks, kThreads, st, e0, e1, a);
}

int launch_distribute(const VerifyArgs& a, void* st, void* e0, void* e1)
{
    return a.dtype == kBF16 ? enqueue(k_distribute<kBF16>, a.blocks, kThreads, st, e0, e1, a)
                            : enqueue(k_distribute<kF32>, a.blocks, kThreads, st, e0, e1, a);
}

int launch_verify_sums(const VerifyArgs& a, void* st, void* e0, void* e1)
{
    if (!a.draft.base && !a.set.top_k && !a.set.top_p && !a.set.min_p) return kNoLaunch;  // (see may_be_many)
    if (a.scan.parts == 0) return kNoLaunch;
    const int64_t items = (int64_t)a.n_seqs * a.ch.max_new;
    const int most = (a.scan.segments + 2 * kScanWaves - 1) / (2 * kScanWaves);
    const int parts = (int)std::max<int64_t>(1, std::min<int64_t>(most, kSumsTarget / std::max<int64_t>(items, 1)));
    const int per = (a.scan.segments + parts - 1) / parts;
    return a.dtype == kBF16 ? enqueue(k_verify_sums<kBF16>, items * parts, kScanThreads, st, e0, e1, a, parts, per)
                            : enqueue(k_verify_sums<kF32>, items * parts, kScanThreads, st, e0, e1, a, parts, per);
}

int launch_verify(const VerifyArgs& a, void* st, void* e0, void* e1)
{
    return a.dtype == kBF16 ? enqueue(k_verify<kBF16>, a.blocks, kThreads, st, e0, e1, a)
                            : enqueue(k_verify<kF32>, a.blocks, kThreads, st, e0, e1, a);
}

int launch_verify_join(const VerifyArgs& a, void* st, void* e0, void* e1)
{
    return enqueue(k_verify_join, (a.n_seqs + 3) / 4, 256, st, e0, e1, a);
}

}  // namespace msao
