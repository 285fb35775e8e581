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
// One workgroup of 1,024 threads has a row. What the settings need decides what it does with it:
//  - one reading for the largest logit of each thread's share, and where every token may
//    stay also the weights' sums over segments of 64 threads' 16 bytes, in the order of the
//    indices and relative to the largest logit of the row's first part;
//  - the head of the order is mostly short. The j-th largest of the 1,024 threads' maxima is a
//    bound that j tokens at least reach and few more, and only the threads whose maximum
//    reaches it read their share again. Up to 1,024 such tokens are ranked in LDS, by
//    comparing each with each, and the row is not read again;
//  - a longer head ends at the key (its logit's bits in order) that histograms of the keys find:
//    2,048 bins between bounds that close in on it, counted, or weighed as integers in two
//    words, so that no order of atomics shows; further readings for what it needs then.
// A weight is 17 instructions of 64 bits (a polynomial of degree 9), which for a row that is
// summed takes about as long as reading it from memory does.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "msao_device.h"
#include "msao_internal.h"
#include "msao_sample.h"

namespace msao {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;

constexpr int kWave = 64;
constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2 * kThreads;
constexpr int kList = kThreads;            // tokens that are ranked in LDS
constexpr int kTryHead = 256;              // of the threads' maxima, for a head whose length top_p decides
constexpr double kLog2e = 1.4426950408889634074;
constexpr double kLn2 = 0.69314718055994530942;
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

// 2^t for t of at most a few hundred: 2^n times a polynomial in t - n, |t - n| <= 1/2. The
// coefficients are those of the interpolation of 2^r at Chebyshev's nodes, with the first one made 1 so that
// equal logits have the weight 1; off by 3.3e-14 of the value at most.
__device__ __forceinline__ double exp2_of(double t)
{
    const double n = __builtin_rint(t), r = t - n;
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
    return __builtin_ldexp(p, (int)n);
}

// Scratch that the steps of a row share.
struct Lds {
    union {
        uint64_t mass[2][kBins];      // a bin's weight in units of 2^-43 and of 2^-86
        uint32_t count[kBins];
        double segment[kMostSegments];
        struct {
            uint64_t packed[kList];   // key, and the index' complement: the order of the tokens, upside down
            double ranked[kList];
        };
    };
    float list_x[kList];              // a head of the order, by index; what does not stay is -inf
    int list_at[kList];
    double wave_d[kWaves];
    int wave_i[kWaves];
    float wave_f[kWaves];
    int wave_b[kWaves];
    double found_d;
    int found_i[3];
};

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

// A row of logits as the workgroup walks it: step i has thread t at the 16 bytes i * kThreads + t,
// so that (step, wavefront, lane) is the order of the indices.
template <int DT>
struct Row {
    static constexpr int N = Chunk<DT>::N, kAhead = 4;
    rsrc_t r;
    int vocab, steps;
    __device__ __forceinline__ Row(const LogitRows& rows, int64_t row, int vocab_) : vocab(vocab_)
    {
        constexpr int es = DT == kBF16 ? 2 : 4;
        // (whole words: a row's pitch is a multiple of 16 bytes)
        r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(rows.base) + row * rows.row_bytes, (short)0,
                                              (vocab * es + 3) & ~3, 0x00020000);
        steps = ((vocab + N - 1) / N + kThreads - 1) / kThreads;
    }
    __device__ __forceinline__ u32x4 load(int chunk) const { return __builtin_amdgcn_raw_buffer_load_b128(r, chunk * 16, 0, 0); }
    __device__ __forceinline__ Chunk<DT> at(int chunk) const
    {
        Chunk<DT> c(load(chunk));
        c.end(vocab - chunk * N);
        return c;
    }
    // f(step, first index, chunk) for every step, by the threads that call it
    template <typename F>
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

// A row's distribution.
struct Dist {
    bool none;        // a NaN, +inf, or no finite logit
    bool listed;      // the tokens that stay are in lds.list, in the order of their indices
    bool summed;      // every token stays, and lds.segment has the sums relative to `ref`
    int best;         // of a row whose largest logit alone stays, its index; else -1
    int kept;         // how many stay where that is known, else -1
    int n;            // entries of the list
    double m, inv;    // largest logit; log2(e) / T
    double ref;
    float cut;        // tokens stay with a logit above it, or equal to it and an index up to cut_at,
    int cut_at;
    double least;     // and (x - m) inv of at least this
    double total;     // of the weights, where it is known
    __device__ __forceinline__ double exponent(float x) const { return ((double)x - m) * inv; }
    __device__ __forceinline__ bool stays(float x, int v) const
    {
        return (x > cut || (x == cut && v <= cut_at)) && exponent(x) >= least;
    }
    __device__ __forceinline__ double weight(float x, int v) const { return stays(x, v) ? exp2_of(exponent(x)) : 0.0; }
};

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

__device__ __forceinline__ double* room_of(Lds& lds, double) { return lds.wave_d; }
__device__ __forceinline__ int* room_of(Lds& lds, int) { return lds.wave_i; }

// Sum over the threads before this one, and the whole. All threads.
template <typename T>
__device__ __forceinline__ T block_before(T v, Lds& lds, T& total)
{
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    T* room = room_of(lds, T(0));
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
    __syncthreads();
    return before + (upto - v);
}

__device__ __forceinline__ double* segments_of(Lds& lds, double) { return lds.segment; }
__device__ __forceinline__ int* segments_of(Lds& lds, int) { return (int*)lds.segment; }

// The sums of f(x, v) >= 0 over the row's segments, in the order of the indices.
template <typename T, int DT, typename F>
__device__ __forceinline__ void sum_segments(const Row<DT>& row, Lds& lds, F f)
{
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    T* segment = segments_of(lds, T(0));
    __syncthreads();
    row.each([&](int i, int v, const Chunk<DT>& c) {
        T s = 0;
#pragma unroll
        for (int e = 0; e < Row<DT>::N; ++e) s += f(c.x[e], v + e);
        s = wave_scan(s);
        if (lane == kWave - 1) segment[i * kWaves + wave] = s;
    });
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
    const int segments = row.steps * kWaves, per = (segments + kThreads - 1) / kThreads;
    const int s0 = min((int)threadIdx.x * per, segments), s1 = min(s0 + per, segments);
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
    // (one atomic a wavefront: most have neither or both)
    const uint64_t hits = __ballot(passed != kNone), any = __ballot(last >= 0);
    if (hits && lane == __builtin_ctzll(hits)) atomicMin(&lds.found_i[0], passed);
    if (any && lane == 63 - __builtin_clzll(any)) atomicMax(&lds.found_i[1], last);
    __syncthreads();
    const int first = lds.found_i[0], s = first != kNone ? first : lds.found_i[1];
    if (first != kNone && passed == first) lds.found_d = (double)base;
    __syncthreads();
    base = (T)lds.found_d;
    if (s >= 0 && wave == 0) {
        const int step = s / kWaves, chunk = step * kThreads + (s - step * kWaves) * kWave + lane;
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
    __syncthreads();
    return locate<T>(row, lds, f, target_of);
}

// Of kBins measures, two a thread from the top down, the first place (from the top) where their running
// sum from `run` on reaches the target, and what lies above it; `last`: of sums that end below it by a
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

// A value that at least j of the threads' values reach and, but for its lower bits, no larger one; -inf where
// there are fewer.
__device__ __forceinline__ float reached_by(Lds& lds, float mine, int j)
{
    const uint32_t k = key_of(mine);
    const bool there = mine > -INFINITY;
    uint32_t prefix = 0;
    double above = 0.0;
#pragma unroll 1
    for (int shift = 21; shift >= 10; shift -= 11) {
        clear_bins(lds, false);
        if (there && (shift == 21 || k >> 21 == prefix >> 21)) atomicAdd(&lds.count[(k >> shift) & (kBins - 1)], 1u);
        __syncthreads();
        const int b0 = kBins - 1 - 2 * (int)threadIdx.x;
        const Place p = top_place(lds, (double)lds.count[b0], (double)lds.count[b0 - 1], above, (double)j, false);
        if (p.at < 0) return -INFINITY;
        prefix |= (uint32_t)(kBins - 1 - p.at) << shift;
        above = p.above;
    }
    return value_of(prefix);
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
    constexpr int N = Row<DT>::N, kUnit = DT == kBF16 ? 16 : 0;  // bf16 values differ in the upper half of their keys
    constexpr double kHi = 8796093022208.0, kInvHi = 1.0 / kHi;  // 2^43
    uint32_t lo = key_of(lowest) >> kUnit, hi = key_of((float)d.m) >> kUnit;
    double above = 0.0;
    bool first = true;
#pragma unroll 1
    while (true) {
        int shift = 0;
        while ((hi - lo) >> shift >= (uint32_t)kBins) ++shift;
        const bool exact = shift == 0;  // a bin is a value: counting weighs it
        clear_bins(lds, MASS && !exact);
        row.each([&](int, int v, const Chunk<DT>& c) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t k = key_of(c.x[e]) >> kUnit;
                if (k < lo || k > hi || !d.stays(c.x[e], v + e)) continue;
                const int bin = (int)((k - lo) >> shift);
                if (MASS && !exact) {
                    const double w = exp2_of(d.exponent(c.x[e])) * kHi;
                    const uint64_t up = (uint64_t)w;
                    atomicAdd((unsigned long long*)&lds.mass[0][bin], up);
                    atomicAdd((unsigned long long*)&lds.mass[1][bin], (uint64_t)((w - (double)up) * kHi));
                } else atomicAdd(&lds.count[bin], 1u);
            }
        });
        __syncthreads();
        // (of a bf16 value the lower half is zeros, of a negative one's key ones)
        auto value = [&](uint32_t k) { return value_of(kUnit && !(k & 0x8000u) ? k << kUnit | 0xFFFFu : k << kUnit); };
        auto measure = [&](int bin) {
            if (!MASS) return (double)lds.count[bin];
            if (!exact) return (double)lds.mass[0][bin] * kInvHi + (double)lds.mass[1][bin] * (kInvHi * kInvHi);
            const uint32_t n = lds.count[bin];
            return n ? (double)n * exp2_of(d.exponent(value(lo + (uint32_t)bin))) : 0.0;
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
            const double w = MASS ? exp2_of(d.exponent(cut.x)) : 1.0, count = (double)lds.count[bin];
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

// The settings of row r.
struct Settings {
    float temperature, top_p, min_p;
    int top_k;
};
__device__ __forceinline__ Settings settings_of(const SamplingDev& s, int r)
{
    return Settings{s.temperature ? s.temperature[r] : 1.0f, s.top_p ? s.top_p[r] : 1.0f, s.min_p ? s.min_p[r] : 0.0f,
                    s.top_k ? s.top_k[r] : 0};
}

// The tokens of `bound` and above in LDS, packed, in an order that is always the same: how many, or more
// than kList, of which none is there. `mine`: the largest logit of the thread's share.
template <int DT>
__device__ __forceinline__ int collect(const Row<DT>& row, Lds& lds, float mine, float bound)
{
    constexpr int N = Row<DT>::N;
    const bool some = mine >= bound && mine > -INFINITY;
    int n = 0, total;
    if (some)
        row.each([&](int, int, const Chunk<DT>& c) {
#pragma unroll
            for (int e = 0; e < N; ++e) n += c.x[e] >= bound && c.x[e] > -INFINITY ? 1 : 0;
        });
    int at = block_before(n, lds, total);
    if (total > kList) return total;
    if (some)
        row.each([&](int, int v, const Chunk<DT>& c) {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (c.x[e] >= bound && c.x[e] > -INFINITY) lds.packed[at++] = (uint64_t)key_of(c.x[e]) << 32 | (uint32_t)~(uint32_t)(v + e);
        });
    if (threadIdx.x == 0 && total < kList) lds.packed[total] = 0;  // (they are read in pairs)
    __syncthreads();
    return total;
}

// With n tokens packed in LDS, which are a head of the order: what of them stays. `whole`: the weight that top_p is
// of, or 0 for that of the first top_k of them. False, and nothing changed, where top_p's head goes on behind them.
template <bool KEEP>
__device__ __forceinline__ bool rank(Lds& lds, Dist& d, const Settings& set, int n, int most, double whole)
{
    const int t = threadIdx.x;
    const bool there = t < n;
    const uint64_t mine = there ? lds.packed[t] : 0;
    int by_key = 0, by_index = 0;
    if (uniform(t & ~(kWave - 1)) < n) {
        for (int j = 0; j < n; j += 2) {
            const uint64_t a = lds.packed[j], b = lds.packed[j + 1 < kList ? j + 1 : j];
            by_key += a > mine ? 1 : 0;
            by_index += (uint32_t)a > (uint32_t)mine ? 1 : 0;
            if (j + 1 < n) {
                by_key += b > mine ? 1 : 0;
                by_index += (uint32_t)b > (uint32_t)mine ? 1 : 0;
            }
        }
    }
    const float x = value_of((uint32_t)(mine >> 32));
    const int at = (int)~(uint32_t)mine;
    const double e = there ? d.exponent(x) : 0.0, w = there ? exp2_of(e) : 0.0;
    if (there) lds.ranked[by_key] = w;
    __syncthreads();
    // thread r has the token of rank r
    const double r_w = t < n && t < most ? lds.ranked[t] : 0.0;
    double sum;
    const double before = block_before(r_w, lds, sum);
    bool in = t < n && t < most;
    if (set.top_p < 1.0f) {
        const double of = whole > 0.0 ? whole : sum, target = (double)set.top_p * of;
        if (whole > 0.0 && sum < target) return false;
        in = in && (t == 0 || before < target);
    }
    // (all of them a head of the order: their number says which)
    int kept;
    (void)block_before(in ? 1 : 0, lds, kept);
    const double least = set.min_p > 0.0f ? fmin(log2((double)set.min_p), 0.0) : -INFINITY;
    const bool stays = there && by_key < kept && e >= least;
    (void)block_before(stays ? 1 : 0, lds, kept);
    (void)block_before(t < kept ? r_w : 0.0, lds, d.total);
    if (stays && by_key == kept - 1) {
        lds.found_d = (double)x;
        lds.found_i[0] = at;
    }
    if (KEEP && there) {
        lds.list_x[by_index] = stays ? x : -INFINITY;
        lds.list_at[by_index] = at;
    }
    __syncthreads();
    d.cut = (float)lds.found_d;
    d.cut_at = lds.found_i[0];
    d.kept = kept;
    d.n = n;
    d.listed = KEEP;
    __syncthreads();
    return true;
}

// KEEP: lds.list may be written.
template <bool KEEP, int DT>
__device__ __forceinline__ Dist solve(const Row<DT>& row, Lds& lds, const Settings& set)
{
    constexpr int N = Row<DT>::N;
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    Dist d;
    d.inv = kLog2e / (double)set.temperature;
    d.cut = -INFINITY;
    d.cut_at = -1;
    d.least = -INFINITY;
    d.listed = d.summed = false;
    d.best = d.kept = -1;
    d.n = 0;
    d.total = d.ref = 0.0;
    const bool greedy = !(set.temperature > 0.0f), by_k = set.top_k > 0 && set.top_k < row.vocab;
    const bool small = row.vocab <= kList;  // every token is ranked
    const bool sums = !greedy && !by_k && !small && (set.top_p < 1.0f || !(set.min_p > 0.0f));

    // the largest logit, of each thread and of all; with the sums relative to the largest of the row's first part
    auto largest = [&](float mine, bool bad, bool& any_bad) {
        float m = mine;
#pragma unroll
        for (int s = 1; s < kWave; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
        const bool b = __ballot(bad) != 0;
        __syncthreads();
        if (lane == 0) {
            lds.wave_f[wave] = m;
            lds.wave_b[wave] = b;
        }
        __syncthreads();
        any_bad = false;
        for (int w = 0; w < kWaves; ++w) {
            m = fmaxf(m, lds.wave_f[w]);
            any_bad = any_bad || lds.wave_b[w] != 0;
        }
        return m;
    };
    float mine = -INFINITY;
    bool bad = false;
    auto look = [&](const Chunk<DT>& c) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            bad = bad || !(c.x[e] < INFINITY);
            mine = fmaxf(mine, c.x[e]);
        }
    };
    if (sums) {
        const Chunk<DT> c = row.at(threadIdx.x);
        float f = -INFINITY;
#pragma unroll
        for (int e = 0; e < N; ++e) f = fmaxf(f, c.x[e]);
        bool ignored;
        f = largest(f, false, ignored);
        d.ref = f > -INFINITY && f < INFINITY ? (double)f : 0.0;
        __syncthreads();
        row.each([&](int i, int, const Chunk<DT>& c) {
            look(c);
            double s = 0.0;
#pragma unroll
            for (int e = 0; e < N; ++e) s += c.x[e] > -INFINITY ? exp2_of(((double)c.x[e] - d.ref) * d.inv) : 0.0;
            s = wave_scan(s);
            if (lane == kWave - 1) lds.segment[i * kWaves + wave] = s;
        });
    } else
        row.each([&](int, int, const Chunk<DT>& c) { look(c); });
    bool any_bad;
    const float m = largest(mine, bad, any_bad);
    d.none = any_bad || m == -INFINITY;
    d.m = m;
    if (d.none) return d;
    if (greedy) {  // the largest alone: the first of equal ones
        if (threadIdx.x == 0) lds.found_i[0] = kNone;
        __syncthreads();
        int at = kNone;
        if (mine == m)
            row.each([&](int, int v, const Chunk<DT>& c) {
#pragma unroll
                for (int e = 0; e < N; ++e) at = c.x[e] == m ? min(at, v + e) : at;
            });
        if (at != kNone) atomicMin(&lds.found_i[0], at);
        __syncthreads();
        d.best = d.cut_at = lds.found_i[0];
        d.inv = 0.0;
        d.cut = m;
        d.kept = 1;
        d.total = 1.0;
        __syncthreads();
        return d;
    }

    const int k = by_k ? set.top_k : row.vocab;
    double whole = 0.0;
    if (sums) {
        auto weigh = [&](float x, int) { return x > -INFINITY ? exp2_of(((double)x - d.ref) * d.inv) : 0.0; };
        if ((d.m - d.ref) * d.inv > 900.0) {  // (sums of such weights may not hold)
            d.ref = d.m;
            sum_segments<double>(row, lds, weigh);
        }
        if (!(set.top_p < 1.0f)) {
            d.summed = true;
            return d;
        }
        __syncthreads();
        double part = 0.0;
        for (int s = threadIdx.x; s < row.steps * kWaves; s += kThreads) part += lds.segment[s];
        (void)block_before(part, lds, whole);
        whole *= exp2_of((d.ref - d.m) * d.inv);
    }
    // a short head: its tokens, or more than kList
    const double target = (double)set.top_p * whole;
    float bound = -INFINITY;
    bool attempt = small;
    if (!small && by_k) {
        bound = reached_by(lds, mine, min(k, kThreads));
        attempt = k <= kThreads;
    } else if (!small && sums) {
        attempt = target < (double)kList;  // (no weight is above 1)
        if (attempt) bound = reached_by(lds, mine, kTryHead);
    } else if (!small) {
        attempt = true;  // min_p alone: the tokens of that weight, and some below it by the rounding of the bound
        bound = (float)(d.m + (log2(fmin((double)set.min_p, 1.0)) - 1e-3) / d.inv);
        bound = bound - fabsf(bound) * 1e-6f;
    }
    if (attempt) {
        const int n = collect(row, lds, mine, bound);
        if (n > 0 && n <= kList && rank<KEEP>(lds, d, set, n, min(k, n), by_k || small || !sums ? 0.0 : whole)) return d;
        __syncthreads();
    }

    // a long one
    auto narrow = [&](const Cut& c) {
        d.cut_at = kNone;
        if (!c.all) {  // the first of the tokens of that value
            const Dist before = d;
            d.cut_at = find_in_order<int>(row, lds, [&](float x, int v) { return x == c.x && before.stays(x, v) ? 1 : 0; },
                                          [&](int) { return (int)c.n - 1; }).at;
        }
        d.cut = c.x;
    };
    if (by_k) {
        const Cut c = cut_of<false>(row, lds, d, bound > -INFINITY && k <= kThreads ? bound : -3.402823466e38f, (double)k);
        if (c.there) narrow(c);
    }
    if (set.top_p < 1.0f) {
        double t = target;
        if (!sums) {
            sum_segments<double>(row, lds, [&](float x, int v) { return d.weight(x, v); });
            __syncthreads();
            double part = 0.0;
            for (int s = threadIdx.x; s < row.steps * kWaves; s += kThreads) part += lds.segment[s];
            (void)block_before(part, lds, whole);
            t = (double)set.top_p * whole;
        }
        // the tokens below a (1 - top_p) / vocab of the whole are less than (1 - top_p) of it together; at
        // least the first stays
        const double share = fmax((1.0 - (double)set.top_p) * whole / (double)row.vocab, 1e-300);
        const double low = d.m + (log2(fmin(share, 1.0)) - 1e-3) / d.inv;
        const float lowest = fmaxf((float)(low - fabs(low) * 1e-6), -3.402823466e38f);
        const Cut c = cut_of<true>(row, lds, d, lowest, fmax(t, 1e-300));
        if (c.there) narrow(c);
    }
    if (set.min_p > 0.0f) d.least = fmin(log2((double)set.min_p), 0.0);
    return d;
}

// u as the running sum's target: [0, 1), NaN as 0.
__device__ __forceinline__ double drawn(float u, double total) { return (u > 0.0f ? (double)u : 0.0) * total; }

// The first token whose running sum of f(x, v) >= 0, 0 of a token that does not stay, passes u times the
// whole; -1 where nothing is.
template <int DT, typename F>
__device__ __forceinline__ Found<double> pick(const Row<DT>& row, Lds& lds, const Dist& d, float u, F f)
{
    if (!d.listed) return find_in_order<double>(row, lds, f, [&](double total) { return drawn(u, total); });
    const int t = threadIdx.x, lane = t & (kWave - 1);
    const float x = t < d.n ? lds.list_x[t] : -INFINITY;
    const double w = x > -INFINITY ? f(x, lds.list_at[t]) : 0.0;
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

// A token of the distribution, with the weights' sum.
template <int DT>
__device__ __forceinline__ Found<double> draw(const Row<DT>& row, Lds& lds, const Dist& d, float u)
{
    if (d.best >= 0) return Found<double>{d.best, 1.0};
    if (d.summed) {
        Found<double> f = locate<double>(row, lds, [&](float x, int) { return x > -INFINITY ? exp2_of(((double)x - d.ref) * d.inv) : 0.0; },
                                         [&](double total) { return drawn(u, total); });
        f.total *= exp2_of((d.ref - d.m) * d.inv);
        // (relative to a smaller logit than the largest a weight may be above 0 that is not)
        if (f.at >= 0 && exp2_of(d.exponent(row.value(f.at))) > 0.0) return f;
    }
    return pick(row, lds, d, u, [&](float x, int v) { return d.weight(x, v); });
}

// The weights' sum alone.
template <int DT>
__device__ __forceinline__ double whole_of(const Row<DT>& row, Lds& lds, const Dist& d)
{
    if (d.best >= 0 || d.kept >= 0) return d.total;
    if (!d.summed) sum_segments<double>(row, lds, [&](float x, int v) { return d.weight(x, v); });
    __syncthreads();
    double part = 0.0, total;
    for (int s = threadIdx.x; s < row.steps * kWaves; s += kThreads) part += lds.segment[s];
    (void)block_before(part, lds, total);
    return d.summed ? total * exp2_of((d.ref - d.m) * d.inv) : total;
}

// ln p of token v.
template <int DT>
__device__ __forceinline__ float logprob_of(const Row<DT>& row, const Dist& d, int v, double total)
{
    return (float)((d.exponent(row.value(v)) - log2(total)) * kLn2);
}

template <int DT>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a)
{
    __shared__ Lds lds;
    const int r = blockIdx.x;
    const Row<DT> row(a.logits, r, a.vocab);
    const Dist d = solve<true>(row, lds, settings_of(a.set, r));
    Found<double> f{-1, 0.0};
    int kept = 0;
    if (!d.none) {
        f = draw(row, lds, d, a.u[r]);
        kept = d.kept;
        if (a.kept && kept < 0) {
            int n = 0;
            row.each([&](int, int v, const Chunk<DT>& c) {
#pragma unroll
                for (int e = 0; e < Row<DT>::N; ++e) n += d.stays(c.x[e], v + e) ? 1 : 0;
            });
            (void)block_before(n, lds, kept);
        }
    }
    if (threadIdx.x != 0) return;
    if (a.token) a.token[r] = f.at;
    if (a.kept) a.kept[r] = kept;
    if (a.logprob) a.logprob[r] = f.at < 0 ? __builtin_nanf("") : logprob_of(row, d, f.at, f.total);
}

// Row i of sequence s: whether its draft stands, and the token that follows it.
template <int DT>
__global__ __launch_bounds__(kThreads) void k_verify(VerifyArgs a)
{
    __shared__ Lds lds;
    const int s = blockIdx.x / a.ch.max_new, i = blockIdx.x - s * a.ch.max_new;
    const Rows rows = seq_rows(a.ch, s);
    const int n = min(rows.n, a.ch.max_new);
    if (i >= n) return;
    const int r = rows.begin + i;
    const bool last = i == n - 1;
    const Row<DT> row(a.logits, r, a.vocab);
    const Settings set = settings_of(a.set, r);
    const Dist p = solve<true>(row, lds, set);
    int token = -1;
    bool yes = false;
    double total = 1.0;
    if (!p.none) {
        const float u = a.u[r];
        if (!last) {
            const int draft = a.tokens[r + 1];
            const bool known = draft >= 0 && draft < a.vocab;
            const double wd = known ? p.weight(row.value(draft), draft) : 0.0;
            const double ua = a.u_accept[r] > 0.0f ? (double)a.u_accept[r] : 0.0;
            total = whole_of(row, lds, p);
            bool certain = a.draft.base == nullptr;
            if (!certain) {
                const Row<DT> other(a.draft, r, a.vocab);
                const Dist q = solve<false>(other, lds, set);
                certain = q.none;
                if (!certain) {
                    const double qt = whole_of(other, lds, q), qd = known ? q.weight(other.value(draft), draft) : 0.0;
                    yes = ua * qd * total < wd * qt;
                    if (!yes)  // what p has more than q
                        token = pick(row, lds, p, u, [&](float x, int v) {
                            const double w = p.weight(x, v);
                            return w > 0.0 ? fmax(w * qt - q.weight(other.value(v), v) * total, 0.0) : 0.0;
                        }).at;
                }
            }
            if (certain) {
                yes = ua * total < wd;
                if (!yes) token = pick(row, lds, p, u, [&](float x, int v) { return v == draft ? 0.0 : p.weight(x, v); }).at;
            }
            if (yes) token = draft;
        }
        if (token < 0) {
            Dist again = p;
            if (!last) again.summed = false;  // (the segments are others' by now)
            const Found<double> f = draw(row, lds, again, u);
            token = f.at;
            total = f.total;
        }
    }
    if (threadIdx.x != 0) return;
    a.row_token[r] = token;
    a.row_yes[r] = yes ? 1 : 0;
    a.row_logprob[r] = token < 0 ? __builtin_nanf("") : logprob_of(row, p, token, total);
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

template <typename K, typename A>
int enqueue(K kernel, int64_t blocks, int threads, void* stream, void* ev0, void* ev1, const A& a)
{
    if (blocks <= 0) return kNoLaunch;
    if (ev0 && ev1)
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, (hipStream_t)stream, (hipEvent_t)ev0, (hipEvent_t)ev1, 0, a);
    else
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}

}  // namespace

int launch_sample(const SampleArgs& a, void* st, void* e0, void* e1)
{
    return a.dtype == kBF16 ? enqueue(k_sample<kBF16>, a.rows, kThreads, st, e0, e1, a)
                            : enqueue(k_sample<kF32>, a.rows, kThreads, st, e0, e1, a);
}

int launch_verify(const VerifyArgs& a, void* st, void* e0, void* e1)
{
    const int64_t blocks = (int64_t)a.n_seqs * a.ch.max_new;
    return a.dtype == kBF16 ? enqueue(k_verify<kBF16>, blocks, kThreads, st, e0, e1, a)
                            : enqueue(k_verify<kF32>, blocks, kThreads, st, e0, e1, a);
}

int launch_verify_join(const VerifyArgs& a, void* st, void* e0, void* e1)
{
    return enqueue(k_verify_join, (a.n_seqs + 3) / 4, 256, st, e0, e1, a);
}

}  // namespace msao
