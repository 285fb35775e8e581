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
// One workgroup of 1,024 threads has a row. The cut of the order is found by the digits of
// the logits' ordered keys (11 bits at a time), counted or weighed in LDS; weights are summed
// there as integers in two words, so that no order of atomics shows.
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
constexpr int kBins = 2048;
constexpr double kLog2e = 1.4426950408889634074;
constexpr double kLn2 = 0.69314718055994530942;
constexpr uint32_t kLowest = 0x007FFFFFu;  // the key of -inf
constexpr int kMostSegments = 4096;        // of a row of kMaxVocab float32 logits

// Keys in the order of the values; +0 and -0 have been made one.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// Scratch that the steps of a row share.
struct Lds {
    union {
        uint64_t mass[2][kBins];      // a bin's weight in units of 2^-43 and of 2^-86
        uint32_t count[kBins];
        double segment[kMostSegments];
    };
    double wave_d[kWaves];
    uint64_t wave_u[kWaves];
    float wave_f[kWaves];
    int wave_i[kWaves];
    double found_d[4];
    int found_i[4];
};

// 16 bytes of a row, widened; what lies past its end, and -inf, is the value that no token has.
template <int DT>
struct Chunk {
    static constexpr int N = DT == kBF16 ? 8 : 4;
    float x[N];
    __device__ __forceinline__ Chunk(const u32x4& w, int n)
    {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if constexpr (DT == kBF16) x[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
            else x[e] = __uint_as_float(w[e]);
            x[e] = e < n ? x[e] + 0.0f : -INFINITY;  // (-0 becomes 0)
        }
    }
};

// A row of logits as the workgroup walks it: step i has thread t at the 16 bytes i * kThreads + t,
// so that (step, wavefront, lane) is the order of the indices.
template <int DT>
struct Row {
    static constexpr int N = Chunk<DT>::N;
    rsrc_t r;
    int vocab, chunks, steps;
    __device__ __forceinline__ Row(const LogitRows& rows, int64_t row, int vocab_) : vocab(vocab_)
    {
        constexpr int es = DT == kBF16 ? 2 : 4;
        // (whole words: a row's pitch is a multiple of 16 bytes)
        r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(rows.base) + row * rows.row_bytes, (short)0,
                                              (vocab * es + 3) & ~3, 0x00020000);
        chunks = (vocab + N - 1) / N;
        steps = (chunks + kThreads - 1) / kThreads;
    }
    __device__ __forceinline__ Chunk<DT> at(int chunk) const
    {
        const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(r, chunk * 16, 0, 0);
        return Chunk<DT>(w, vocab - chunk * N);
    }
    // f(step, first index, chunk) for every step, by all threads
    template <typename F>
    __device__ __forceinline__ void each(F f) const
    {
        for (int i = 0; i < steps; ++i) {
            const int c = i * kThreads + threadIdx.x;
            f(i, c * N, at(c));
        }
    }
    __device__ __forceinline__ float value(int v) const
    {
        if constexpr (DT == kBF16) return __uint_as_float((uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, 2 * v, 0, 0) << 16) + 0.0f;
        return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, 4 * v, 0, 0)) + 0.0f;
    }
};

// A row's distribution.
struct Dist {
    bool none;        // a NaN, +inf, or no finite logit
    int best;         // index of the largest, the first of equal ones
    double m, inv;    // largest logit; log2(e) / T
    uint32_t cut;     // tokens stay with a key above it, or of it and an index up to cut_at,
    int cut_at;
    double least;     // and (x - m) inv of at least this
    __device__ __forceinline__ double exponent(float x) const { return ((double)x - m) * inv; }
    __device__ __forceinline__ bool stays(float x, int v) const
    {
        const uint32_t k = key_of(x);
        return (k > cut || (k == cut && v <= cut_at)) && exponent(x) >= least;
    }
    __device__ __forceinline__ double weight(float x, int v) const { return stays(x, v) ? exp2(exponent(x)) : 0.0; }
};

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) v += __shfl_xor(v, s);
    return v;
}

// Sums of the lanes up to each, by T.
template <typename T>
__device__ __forceinline__ T wave_scan(T v)
{
    const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
        const T o = __shfl_up(v, s);
        if (lane >= s) v += o;
    }
    return v;
}

// Sum over the threads before this one, and the whole. All threads; `room` is free afterwards.
template <typename T>
__device__ __forceinline__ T block_before(T v, T* room, T& total)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
    const T upto = wave_scan(v);
    if (lane == kWave - 1) room[wave] = upto;
    __syncthreads();
    T before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        before += w < wave ? room[w] : T(0);
        total += room[w];
    }
    __syncthreads();
    const T up = __shfl_up(upto, 1);
    return before + (lane > 0 ? up : T(0));
}

__device__ __forceinline__ int block_sum(int v, Lds& lds)
{
    int total;
    block_before(v, lds.wave_i, total);
    return total;
}

// The first index whose running sum of f(x, v) >= 0 passes target(total), in the order of the
// indices; the last one with f > 0 where none does, -1 where there is none. Every thread gets it.
struct Found {
    int at;
    double total;
};
template <int DT, typename F, typename T>
__device__ __forceinline__ Found find_in_order(const Row<DT>& row, Lds& lds, F f, T target_of)
{
    constexpr int N = Row<DT>::N;
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    __syncthreads();
    if (threadIdx.x == 0) {
        lds.found_i[0] = 0x7FFFFFFF;
        lds.found_i[1] = -1;
    }
    row.each([&](int i, int v, const Chunk<DT>& c) {
        double s = 0.0;
#pragma unroll
        for (int e = 0; e < N; ++e) s += f(c.x[e], v + e);
        s = wave_sum(s);
        if (lane == 0) lds.segment[i * kWaves + wave] = s;
    });
    __syncthreads();
    const int segments = row.steps * kWaves, per = (segments + kThreads - 1) / kThreads;
    const int s0 = min((int)threadIdx.x * per, segments), s1 = min(s0 + per, segments);
    double mine = 0.0;
    for (int s = s0; s < s1; ++s) mine += lds.segment[s];
    double total;
    const double before = block_before(mine, lds.wave_d, total);
    const double target = target_of(total);
    // the first segment that passes the target, or the last one that has anything (the sums of
    // neighbouring threads may overlap or leave a gap by a rounding)
    double run = before, base = 0.0;
    int passed = 0x7FFFFFFF;
    for (int s = s0; s < s1; ++s) {
        const double w = lds.segment[s];
        if (w > 0.0) {
            if (passed == 0x7FFFFFFF && run + w > target) {
                passed = s;
                base = run;
            }
            atomicMax(&lds.found_i[1], s);
        }
        run += w;
    }
    if (passed != 0x7FFFFFFF) atomicMin(&lds.found_i[0], passed);
    __syncthreads();
    const int first = lds.found_i[0], s = first != 0x7FFFFFFF ? first : lds.found_i[1];
    if (passed == first && first != 0x7FFFFFFF) lds.found_d[0] = base;
    __syncthreads();
    base = lds.found_d[0];
    if (s >= 0 && wave == 0) {
        const int step = s / kWaves, chunk = step * kThreads + (s - step * kWaves) * kWave + lane;
        const Chunk<DT> c = row.at(chunk);
        double w[N], sum = 0.0;
        int top = -1;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            w[e] = f(c.x[e], chunk * N + e);
            sum += w[e];
            if (w[e] > 0.0) top = e;
        }
        const double r = base + (wave_scan(sum) - sum);
        int at = -1;
#pragma unroll
        for (int e = N - 1; e >= 0; --e) {
            double upto = r;
#pragma unroll
            for (int q = 0; q <= e; ++q) upto += w[q];
            if (w[e] > 0.0 && upto > target) at = e;  // the first at the end
        }
        const uint64_t hit = first != 0x7FFFFFFF ? __ballot(at >= 0) : 0, any = __ballot(top >= 0);
        const int winner = hit ? __builtin_ctzll(hit) : any ? 63 - __builtin_clzll(any) : 0;
        if (lane == winner) lds.found_i[2] = chunk * N + (hit ? at : top);
    }
    __syncthreads();
    const Found out{s >= 0 ? lds.found_i[2] : -1, total};
    __syncthreads();
    return out;
}

// The key at which the measure of the tokens that stay in d, summed down the order, reaches
// target(total); what lies above it.
struct Cut {
    bool there;
    uint32_t key;
    double above, target;
};
// (a weight is at most 1 and a row has at most 2^20: 2^43 of them stay below 2^63)
template <bool MASS, int DT, typename T>
__device__ __forceinline__ Cut cut_of(const Row<DT>& row, Lds& lds, const Dist& d, T target_of)
{
    constexpr int N = Row<DT>::N;
    constexpr double kHi = 8796093022208.0, kInvHi = 1.0 / kHi;  // 2^43
    Cut cut{false, 0, 0.0, 0.0};
    uint32_t prefix = 0, mask = 0;
    // bf16 values differ in the upper 16 bits of their keys
#pragma unroll 1
    for (int shift = 21; shift >= (DT == kBF16 ? 10 : 0); shift -= shift == 10 ? 10 : 11) {
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += kThreads) {
            if (MASS) lds.mass[0][b] = lds.mass[1][b] = 0;
            else lds.count[b] = 0;
        }
        __syncthreads();
        row.each([&](int, int v, const Chunk<DT>& c) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t k = key_of(c.x[e]);
                if ((k & mask) != prefix || !d.stays(c.x[e], v + e)) continue;
                const int bin = (k >> shift) & (kBins - 1);
                if (MASS) {
                    const double w = exp2(d.exponent(c.x[e])) * kHi;
                    const uint64_t hi = (uint64_t)w;
                    atomicAdd((unsigned long long*)&lds.mass[0][bin], hi);
                    atomicAdd((unsigned long long*)&lds.mass[1][bin], (uint64_t)((w - (double)hi) * kHi));
                } else atomicAdd(&lds.count[bin], 1u);
            }
        });
        __syncthreads();
        // two bins a thread, the upper ones first
        const int b0 = kBins - 1 - 2 * (int)threadIdx.x;
        double m[2];
#pragma unroll
        for (int q = 0; q < 2; ++q)
            m[q] = MASS ? (double)lds.mass[0][b0 - q] * kInvHi + (double)lds.mass[1][b0 - q] * (kInvHi * kInvHi)
                        : (double)lds.count[b0 - q];
        if (threadIdx.x == 0) {
            lds.found_i[0] = kBins;
            lds.found_i[1] = -1;
        }
        double total, run = cut.above + block_before(m[0] + m[1], lds.wave_d, total);
        if (mask == 0) cut.target = target_of(total);
        // the first bin that reaches the target; of a later level, whose sums may end below it by a
        // rounding, else the last one that has anything. Places count from the top
        int place = kBins, last = -1;
        double above = 0.0;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (m[q] > 0.0) {
                last = kBins - 1 - b0 + q;
                if (place == kBins && run + m[q] >= cut.target) {
                    place = last;
                    above = run;
                }
            }
            run += m[q];
        }
        if (place != kBins) atomicMin(&lds.found_i[0], place);
        if (last >= 0) atomicMax(&lds.found_i[1], last);
        __syncthreads();
        const int reached = lds.found_i[0], at = reached != kBins ? reached : mask != 0 ? lds.found_i[1] : -1;
        if (at < 0) return cut;
        const int mine = at - 2 * (int)threadIdx.x;
        if (mine == 0 || mine == 1) lds.found_d[0] = reached != kBins ? above : run - (mine == 0 ? m[0] + m[1] : m[1]);
        __syncthreads();
        const int bin = kBins - 1 - at;
        cut.above = lds.found_d[0];
        prefix |= (uint32_t)bin << shift;
        mask |= (uint32_t)(kBins - 1) << shift;
    }
    cut.there = true;
    // (of a bf16 value the lower bits are zeros, of a negative one's key ones)
    cut.key = prefix;
    if (DT == kBF16 && !(prefix & 0x80000000u)) cut.key |= 0x3FF;
    return cut;
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

template <int DT>
__device__ __forceinline__ Dist solve(const Row<DT>& row, Lds& lds, const Settings& set)
{
    constexpr int N = Row<DT>::N;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
    Dist d;
    float m = -INFINITY;
    int best = 0x7FFFFFFF;
    bool bad = false;
    row.each([&](int, int v, const Chunk<DT>& c) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            bad = bad || !(c.x[e] < INFINITY);
            if (c.x[e] > m) {
                m = c.x[e];
                best = v + e;
            }
        }
    });
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
        const float om = __shfl_xor(m, s);
        const int ob = __shfl_xor(best, s);
        if (om > m || (om == m && ob < best)) {
            m = om;
            best = ob;
        }
    }
    bad = __ballot(bad) != 0;
    if (lane == 0) {
        lds.wave_f[wave] = m;
        lds.wave_i[wave] = best;
        lds.wave_u[wave] = bad;
    }
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
        const float om = lds.wave_f[w];
        const int ob = lds.wave_i[w];
        bad = bad || lds.wave_u[w] != 0;
        if (om > m || (om == m && ob < best)) {
            m = om;
            best = ob;
        }
    }
    __syncthreads();
    d.none = bad || m == -INFINITY;
    d.best = best;
    d.m = m;
    d.inv = kLog2e / (double)set.temperature;
    d.cut = kLowest;
    d.cut_at = -1;
    d.least = -INFINITY;
    if (d.none) return d;
    if (!(set.temperature > 0.0f)) {  // the largest alone
        d.inv = 0.0;
        d.cut = key_of(m);
        d.cut_at = best;
        return d;
    }
    auto narrow = [&](uint32_t key, double n) {  // the first n of the tokens of that key
        const Found f = find_in_order<DT>(row, lds, [&](float x, int v) { return key_of(x) == key && d.stays(x, v) ? 1.0 : 0.0; },
                                          [&](double) { return n - 1.0; });
        d.cut = key;
        d.cut_at = f.at;
    };
    if (set.top_k > 0 && set.top_k < row.vocab) {
        const Cut c = cut_of<false, DT>(row, lds, d, [&](double) { return (double)set.top_k; });
        if (c.there) narrow(c.key, (double)set.top_k - c.above);
    }
    if (set.top_p < 1.0f) {
        // (at least the first token; sums that are 0 throughout cannot be)
        const Cut c = cut_of<true, DT>(row, lds, d, [&](double total) { return fmax((double)set.top_p * total, 1e-300); });
        if (c.there) {
            const double w = exp2(d.exponent(value_of(c.key)));
            double n = fmax(ceil((c.target - c.above) / w), 1.0);
            if (n > 1.0 && c.above + (n - 1.0) * w >= c.target) n -= 1.0;
            narrow(c.key, n);
        }
    }
    if (set.min_p > 0.0f) d.least = fmin(log2((double)set.min_p), 0.0);
    return d;
}

// u as the running sum's target: [0, 1), NaN as 0.
__device__ __forceinline__ double drawn(float u, double total) { return (u > 0.0f ? (double)u : 0.0) * total; }

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
    const Dist d = solve(row, lds, settings_of(a.set, r));
    Found f{-1, 0.0};
    int kept = 0;
    if (!d.none) {
        const float u = a.u[r];
        f = find_in_order<DT>(row, lds, [&](float x, int v) { return d.weight(x, v); }, [&](double total) { return drawn(u, total); });
        if (a.kept) {
            int n = 0;
            row.each([&](int, int v, const Chunk<DT>& c) {
#pragma unroll
                for (int e = 0; e < Row<DT>::N; ++e) n += d.stays(c.x[e], v + e) ? 1 : 0;
            });
            kept = block_sum(n, lds);
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
    const Dist p = solve(row, lds, set);
    int token = -1;
    bool yes = false;
    double total = 0.0;
    if (!p.none) {
        const int draft = last ? -1 : a.tokens[r + 1];
        const bool known = draft >= 0 && draft < a.vocab;
        const float u = a.u[r];
        auto weight = [&](float x, int v) { return p.weight(x, v); };
        auto plain = [&]() { return find_in_order<DT>(row, lds, weight, [&](double t) { return drawn(u, t); }); };
        Found f = plain();
        total = f.total;
        token = f.at;
        if (!last) {
            const double wd = known ? p.weight(row.value(draft), draft) : 0.0;
            const double ua = a.u_accept[r] > 0.0f ? (double)a.u_accept[r] : 0.0;
            bool certain = a.draft.base == nullptr;
            if (!certain) {
                const Row<DT> other(a.draft, r, a.vocab);
                const Dist q = solve(other, lds, set);
                certain = q.none;
                if (!certain) {
                    const double qt = find_in_order<DT>(other, lds, [&](float x, int v) { return q.weight(x, v); }, [](double) { return 0.0; }).total;
                    const double qd = known ? q.weight(other.value(draft), draft) : 0.0;
                    yes = ua * qd * total < wd * qt;
                    if (!yes) {
                        // what p has more than q
                        f = find_in_order<DT>(row, lds,
                                              [&](float x, int v) {
                                                  const double w = p.weight(x, v);
                                                  return w > 0.0 ? fmax(w * qt - q.weight(other.value(v), v) * total, 0.0) : 0.0;
                                              },
                                              [&](double t) { return drawn(u, t); });
                        if (f.at >= 0) token = f.at;
                    }
                }
            }
            if (certain) {
                yes = ua * total < wd;
                if (!yes) {
                    f = find_in_order<DT>(row, lds, [&](float x, int v) { return v == draft ? 0.0 : p.weight(x, v); },
                                          [&](double t) { return drawn(u, t); });
                    if (f.at >= 0) token = f.at;
                }
            }
            if (yes) token = draft;
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
