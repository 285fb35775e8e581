// msao_cache.hip -- gfx950 (CDNA4) kernels that store to a paged cache: append (norm of
// the queries' and keys' heads, position rotation, and the keys and values into their
// pages, in one pass) and eviction by accumulated attention weight.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "msao_cache.h"
#include "msao_device.h"
#include "msao_internal.h"

namespace msao {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kWave = 64;
constexpr int kBlock = 256;
constexpr int kWaves = kBlock / kWave;
constexpr int kMaxPairs = 128;  // of a rotation: half the largest head

// Eight neighbouring values of a row in 32 bits.
template <int DT>
struct Eight {
    u32x4 w[DT == kBF16 ? 1 : 2];
    __device__ __forceinline__ void load(const uint8_t* p)
    {
        w[0] = ((const u32x4*)p)[0];
        if constexpr (DT == kF32) w[1] = ((const u32x4*)p)[1];
    }
    __device__ __forceinline__ void store(uint8_t* p) const
    {
        ((u32x4*)p)[0] = w[0];
        if constexpr (DT == kF32) ((u32x4*)p)[1] = w[1];
    }
    __device__ __forceinline__ void zero()
    {
        w[0] = u32x4{0, 0, 0, 0};
        if constexpr (DT == kF32) w[1] = w[0];
    }
    __device__ __forceinline__ void widen(float (&x)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (DT == kBF16) {
                x[2 * e] = __uint_as_float(w[0][e] << 16);
                x[2 * e + 1] = __uint_as_float(w[0][e] & 0xFFFF0000u);
            } else {
                x[e] = __uint_as_float(w[0][e]);
                x[4 + e] = __uint_as_float(w[1][e]);
            }
        }
    }
    __device__ __forceinline__ void narrow(const float (&x)[8])
    {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (DT == kBF16) {
                const f32x2 v = {x[2 * e], x[2 * e + 1]};
                w[0][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf2));
            } else {
                w[0][e] = __float_as_uint(x[e]);
                w[1][e] = __float_as_uint(x[4 + e]);
            }
        }
    }
};

// The sequence of a row of the chunk (-1: none), and its rows: the first sequence whose rows
// (seq_rows) the row is one of, 64 sequences at a time. `first`, `last`: the lane's starts and
// ends of the first 64.
__device__ __forceinline__ int seq_of_row(const AppendArgs& a, int row, int first, int last, Rows* rows)
{
    const int lane = threadIdx.x & (kWave - 1);
    for (int s0 = 0; s0 < a.c.n_seqs; s0 += kWave) {
        const int s = s0 + lane;
        if (s0 > 0) {
            first = a.ch.start[min(s, a.c.n_seqs)];
            last = a.ch.start[min(s + 1, a.c.n_seqs)];
        }
        const int b = clamp_int(first, 0, a.ch.n_rows), e = clamp_int(last, b, a.ch.n_rows);
        const uint64_t mine = __ballot(s < a.c.n_seqs && row >= b && row < e);
        if (mine == 0) continue;
        const int at = __builtin_ctzll(mine);
        rows->begin = __builtin_amdgcn_readlane(b, at);
        rows->n = __builtin_amdgcn_readlane(e, at) - rows->begin;
        return s0 + at;
    }
    return -1;
}

// One pass over a row's heads: queries, keys, then values. A head takes `lanes` lanes of
// a wavefront (a power of two), each with two eights of it that hold whole pairs of the
// rotation: (8u, rot/2 + 8u) below rot (or 16u, 16u + 8 for neighbouring pairs), two
// neighbours above. The norm is a sum over those lanes; the angles are the same for
// every head, so a wavefront computes each once, into LDS, and a lane keeps the eight
// that it turns. HBM bound: each value is read and written once, four heads in flight.
// The angle is taken in turns in 64 bits (position * inv_freq / 2 pi), less its quarter
// turns, which keeps far positions as exact as near ones and rounds at most an eighth of a
// turn to 32 bits: 2^-28 of a turn, 2.3e-8 rad, where a whole turn's 2^-25 is three steps of a sine below 1.
template <int DT>
__global__ __launch_bounds__(kBlock) void k_append(AppendArgs a)
{
    constexpr int ES = DT == kBF16 ? 2 : 4;
    constexpr int U = 4;  // rounds of heads in flight
    __shared__ f32x2 turn[kWaves][kMaxPairs];
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    const uint32_t item = blockIdx.x * kWaves + wave;  // below 2^27
    const int row = item / (uint32_t)a.parts, part = item - row * a.parts;
    if (row >= a.ch.n_rows) return;
    const int u = lane & (a.lanes - 1), per = kWave / a.lanes;  // the lane's pair of eights; heads of a round
    const int half = a.rot / 2, turned = a.rot / 16;
    const bool turns = u < turned;
    int d0, d1;
    if (turns && !a.neighbours) {
        d0 = 8 * u;
        d1 = half + 8 * u;
    } else {
        d0 = 16 * u;
        d1 = d0 + 8;
    }
    const bool has0 = d0 < a.c.dim, has1 = d1 < a.c.dim;
    const int heads = a.heads + 2 * a.c.kv_heads;
    const int rounds = (heads + per - 1) / per;
    Eight<DT> x0[U], x1[U];
    auto load = [&](int r0) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int h = (r0 + j) * per + lane / a.lanes;
            x0[j].zero();
            x1[j].zero();
            if (h >= heads) continue;
            const uint8_t* src;
            if (h < a.heads) src = a.q + row * a.q_stride + (int64_t)h * a.c.dim * ES;
            else if (h < a.heads + a.c.kv_heads) src = a.k + row * a.k_stride + (int64_t)(h - a.heads) * a.c.dim * ES;
            else src = a.v + row * a.v_stride + (int64_t)(h - a.heads - a.c.kv_heads) * a.c.dim * ES;
            if (has0) x0[j].load(src + d0 * ES);
            if (has1) x1[j].load(src + d1 * ES);
        }
    };
    // what needs no sequence is on its way while the row's sequence, place and page are found
    const int first = a.ch.start[min(lane, a.c.n_seqs)], last = a.ch.start[min(lane + 1, a.c.n_seqs)];
    int at[2] = {0, 0};
    float freq[2] = {0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int i = lane + kWave * e;
        if (i >= half) continue;
        int axis = 0;
#pragma unroll
        for (int x = 0; x < 3; ++x) axis += i >= a.axis_end[x];
        if (a.positions) at[e] = a.positions[axis * a.position_stride + row];
        freq[e] = a.inv_freq[i];
    }
    load(part * U);
    Eight<DT> nq0, nq1, nk0, nk1;
    nq0.zero();
    nq1.zero();
    nk0.zero();
    nk1.zero();
    if (a.q_norm && has0) nq0.load(a.q_norm + d0 * ES);
    if (a.q_norm && has1) nq1.load(a.q_norm + d1 * ES);
    if (a.k_norm && has0) nk0.load(a.k_norm + d0 * ES);
    if (a.k_norm && has1) nk1.load(a.k_norm + d1 * ES);
    Rows rows;
    const int s = uniform(seq_of_row(a, row, first, last, &rows));
    if (s < 0) return;
    const int64_t place = (int64_t)seq_length(a.c, s) - rows.n + (row - rows.begin);  // in the cache
    const int mask = (1 << a.c.page_shift) - 1;
    const int page = place >= 0 ? page_at(a.c, s, (int)place >> a.c.page_shift) : -1;
    const int slot = (int)place & mask;

#pragma unroll
    for (int e = 0; e < 2; ++e) {
        if (kWave * e >= half) break;
        double t = (double)(a.positions ? at[e] : (int)place) * (double)freq[e] * 0.15915494309189533577;
        const double quarters = rint(4.0 * t);
        t -= 0.25 * quarters;  // exact, in [-1/8, 1/8]
        float sn, cs;
        sincospif(2.0f * (float)t, &sn, &cs);
        const int quarter = (int)(quarters - 4.0 * floor(0.25 * quarters));  // 0 .. 3, of any number of them
        const float x = quarter & 1 ? sn : cs, y = quarter & 1 ? cs : sn;
        const bool minus_x = quarter == 1 || quarter == 2, minus_y = quarter >= 2;
        if (lane + kWave * e < half) turn[wave][lane + kWave * e] = f32x2{minus_x ? -x : x, minus_y ? -y : y};
    }
    // the wavefront's own stores, read by its other lanes
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    float cs[8], sn[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const f32x2 v = turns ? turn[wave][8 * u + e] : f32x2{1.0f, 0.0f};
        cs[e] = v.x;
        sn[e] = v.y;
    }

    if (a.c.weight && part == 0 && place >= 0)
        for (int h = lane; h < a.c.kv_heads; h += kWave)
            a.c.weight[((int64_t)s * a.c.kv_heads + h) * a.c.weight_stride + place] = 0.0f;
    for (int r0 = part * U; r0 < rounds; r0 += a.parts * U) {
        if (r0 != part * U) load(r0);
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int h = (r0 + j) * per + lane / a.lanes;
            const bool is_q = h < a.heads, is_v = h >= a.heads + a.c.kv_heads;
            float y0[8], y1[8];
            x0[j].widen(y0);
            x1[j].widen(y1);
            float sq = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sq = fmaf(y0[e], y0[e], fmaf(y1[e], y1[e], sq));
            for (int o = 1; o < a.lanes; o <<= 1) sq += __shfl_xor(sq, o);
            const uint8_t* norm = is_q ? a.q_norm : a.k_norm;
            if (!is_v) {
                if (norm) {
                    const float f = 1.0f / sqrtf(sq / (float)a.c.dim + a.eps);
                    float w0[8], w1[8];
                    Eight<DT> n0 = nk0, n1 = nk1;
                    if (is_q) {
                        n0 = nq0;
                        n1 = nq1;
                    }
                    n0.widen(w0);
                    n1.widen(w1);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        y0[e] *= f * w0[e];
                        y1[e] *= f * w1[e];
                    }
                }
                if (turns) {
                    if (a.neighbours) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float p = y0[2 * e], q = y0[2 * e + 1], r = y1[2 * e], t = y1[2 * e + 1];
                            y0[2 * e] = p * cs[e] - q * sn[e];
                            y0[2 * e + 1] = p * sn[e] + q * cs[e];
                            y1[2 * e] = r * cs[4 + e] - t * sn[4 + e];
                            y1[2 * e + 1] = r * sn[4 + e] + t * cs[4 + e];
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float p = y0[e], q = y1[e];
                            y0[e] = p * cs[e] - q * sn[e];
                            y1[e] = p * sn[e] + q * cs[e];
                        }
                    }
                }
                x0[j].narrow(y0);
                x1[j].narrow(y1);
            }
            if (h >= heads) continue;
            uint8_t* dst;
            if (is_q) {
                dst = a.q_out + row * a.q_out_stride + (int64_t)h * a.c.dim * ES;
            } else {
                if (page < 0) continue;
                const int kh = is_v ? h - a.heads - a.c.kv_heads : h - a.heads;
                dst = is_v ? a.c.v + page * a.c.v_page + kh * a.c.v_head + slot * a.c.v_tok
                           : a.c.k + page * a.c.k_page + kh * a.c.k_head + slot * a.c.k_tok;
            }
            if (has0) x0[j].store(dst + d0 * ES);
            if (has1) x1[j].store(dst + d1 * ES);
        }
    }
}

// ---- eviction -------------------------------------------------------------------

// The tokens that stay of one (sequence, kv head), by one workgroup: the key of the last
// ranked one by digits of 11, 10 and 10 bits (the sign is 0), counted in LDS, then the kept
// indices and weights in one ascending pass. k_select holds the weights in registers, item i
// of thread t token i T + t, so that loads and stores are of neighbours; in the ascending
// pass each wavefront's counts of each item meet in LDS once, and ballots order the rest.
// Beyond kSelTokens tokens k_select_long goes over memory again for each digit. Bound by
// latency: one pass over the weights and a dozen barriers (8 x 2,944 tokens 12-13 us, 256 x 8,000
// 17-18; 12 x 81,000, past the registers, 73-82).
constexpr int kSelLong = 1024;                    // threads of k_select_long
constexpr int kSelItems = 32;                     // tokens of a thread, at most (64 spill)
constexpr int kSelTokens = kSelItems * kSelLong;
constexpr int kDigits = 3;
__device__ constexpr int kShift[kDigits] = {20, 10, 0}, kWidth[kDigits] = {11, 10, 10};
constexpr int kBins = 2048 + 1024 + 1024;
__device__ __forceinline__ constexpr int first_bin(int d) { return d == 0 ? 0 : 1024 + 1024 * d; }

// Order of a weight: larger is kept; NaN and what is not above 0 counts as 0.
__device__ __forceinline__ uint32_t weight_key(float w) { return w > 0.0f ? __float_as_uint(w) : 0u; }

// Which tokens stay: the first `lo`, those from `hi` on, and `take` of those between.
struct Kept {
    int L, k, lo, hi, take;
    __device__ __forceinline__ Kept(const EvictArgs& a, int s)
    {
        L = seq_length(a.from, s);
        k = min(min(L, max(entry(a.budget, s), 0)), capacity(a.to));
        lo = min(a.n_first, k);
        const int recent = min(a.n_recent, k - lo);
        hi = L - recent;
        take = k - lo - recent;
    }
    __device__ __forceinline__ bool all() const { return take >= hi - lo; }
};

// The least key that stays and how many of that key do; `whole`: all of them from `least` on.
struct Border {
    uint32_t least, ties;
    bool whole;
    __device__ __forceinline__ bool above(uint32_t key) const { return whole ? key >= least : key > least; }
    __device__ __forceinline__ bool equal(uint32_t key) const { return !whole && key == least; }
};

// The bin, from the largest down, in which the `want`-th key lies, the rank within it, and
// its count; every wavefront finds it for itself.
struct Found {
    uint32_t bin, rank, count;
};
template <int BINS>
__device__ __forceinline__ Found find_bin(const uint32_t* bins, uint32_t want)
{
    constexpr int N = BINS / kWave;  // a lane's bins, those of lane 0 the largest
    const int lane = threadIdx.x & (kWave - 1);
    const uint32_t* mine = bins + BINS - (lane + 1) * N;
    uint32_t sum = 0;
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const u32x4 v = *(const u32x4*)(mine + i);
        sum += v[0] + v[1] + v[2] + v[3];
    }
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t y = (uint32_t)__shfl_up((int)upto, o);
        if (lane >= o) upto += y;
    }
    const int at = __builtin_ctzll(__ballot(upto >= want) | 1ull << (kWave - 1));
    const uint32_t before = (uint32_t)__builtin_amdgcn_readlane((int)(upto - sum), at);
    // the N bins of lane `at`, one a lane
    const int top = BINS - 1 - at * N;
    uint32_t c = lane < N ? bins[top - lane] : 0u, run = c;
#pragma unroll
    for (int o = 1; o < N; o <<= 1) {
        const uint32_t y = (uint32_t)__shfl_up((int)run, o);
        if (lane >= o) run += y;
    }
    const int l = __builtin_ctzll(__ballot(lane < N && before + run >= want) | 1ull << (N - 1));
    const uint32_t count = (uint32_t)__builtin_amdgcn_readlane((int)c, l);
    return Found{(uint32_t)(top - l), want - before - ((uint32_t)__builtin_amdgcn_readlane((int)run, l) - count), count};
}

// One digit of the border: its bins are counted; false once the border is known.
template <int D>
__device__ __forceinline__ bool next_digit(Border& b, uint32_t& want, const uint32_t* bins)
{
    const Found f = find_bin<1 << kWidth[D]>(bins + first_bin(D), want);
    b.least |= f.bin << kShift[D];
    want = f.rank;
    b.ties = want;
    b.whole = f.rank == f.count;  // all of the bin stay, whatever the lower digits
    return !b.whole;
}

// Exclusive sum over the block of a per-thread value, and the total.
template <int WAVES>
__device__ __forceinline__ uint64_t block_scan(uint64_t v, uint64_t* lds, uint64_t* total)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
    uint64_t x = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const uint64_t y = (uint64_t)__shfl_up((unsigned long long)x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();  // (an earlier call's sums have been read)
    if (lane == kWave - 1) lds[wave] = x;
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const uint64_t t = lds[w];
        before += w < wave ? t : 0;
        all += t;
    }
    *total = all;
    return before + x - v;
}

// The kept ones of T N tokens from j0 on (v: item i of thread t is token j0 + i T + t; a
// barrier stands between their loads and here): indices and weights to their places.
// `done` (tokens kept beside the ties << 32 | tokens of the border's key before) moves on.
template <int T, int N>
__device__ __forceinline__ void put_kept(const EvictArgs& a, const Kept& q, const Border& b, int sh, int j0, const float (&v)[N],
                                         uint64_t* counts, uint64_t* sums, uint64_t* done, int* moved)
{
    constexpr int W = T / kWave;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = uniform(tid >> 6);
    int32_t* idx = a.kept_idx + (int64_t)sh * a.idx_stride;
    float* tw = a.to.weight ? a.to.weight + (int64_t)sh * a.to.weight_stride : nullptr;
    auto look = [&](int i, uint64_t* above, uint64_t* equal) {
        const int j = j0 + i * T + tid;
        const uint32_t key = weight_key(v[i]);
        const bool there = j < q.L, fixed = j < q.lo || j >= q.hi;
        *above = __ballot(there && (fixed || b.above(key)));
        *equal = __ballot(there && !fixed && b.equal(key));
    };
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint64_t n, e;
        look(i, &n, &e);
        if (lane == 0) counts[i * W + wave] = (uint64_t)__popcll(n) << 32 | (uint32_t)__popcll(e);
    }
    __syncthreads();
    const uint64_t mine = tid < N * W ? counts[tid] : 0;
    uint64_t total;
    const uint64_t before = block_scan<W>(mine, sums, &total);
    if (tid < N * W) counts[tid] = *done + before;
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint64_t n, e;
        look(i, &n, &e);
        const uint64_t base = counts[i * W + wave];
        const uint32_t n_at = (uint32_t)(base >> 32) + __popcll(n & below), e_at = (uint32_t)base + __popcll(e & below);
        if ((n >> lane & 1) || ((e >> lane & 1) && e_at < b.ties)) {
            const int j = j0 + i * T + tid, to = (int)(n_at + min(e_at, b.ties));
            idx[to] = j;
            if (tw) tw[to] = v[i];
            if (to != j) *moved = min(*moved, to);
        }
    }
    *done += total;
}

template <int T>
__device__ __forceinline__ void finish(const EvictArgs& a, const Kept& q, int sh, int moved, int* first_moved)
{
    if (moved < INT32_MAX) atomicMin(first_moved, moved);
    int32_t* idx = a.kept_idx + (int64_t)sh * a.idx_stride;
    const int cap = capacity(a.from);
    for (int j = q.k + (int)threadIdx.x; j < cap; j += T) idx[j] = -1;
    __syncthreads();
    if (threadIdx.x == 0) a.info[sh] = EvictInfo{q.k, a.in_place ? *first_moved : 0};
}

// The border over the tokens that `each` hands to a function one by one (the same ones each time).
template <typename Each>
__device__ __forceinline__ Border find_border(const Kept& q, uint32_t* bins, Each each)
{
    Border border{0, 0, true};  // all stay
    if (q.all()) return border;
    border = Border{q.take > 0 ? 0u : ~0u, 0, false};
    uint32_t want = (uint32_t)max(q.take, 0);
    auto count = [&](auto digit) {
        constexpr int D = decltype(digit)::value;
        __syncthreads();
        each([&](int j, float w) {
            const uint32_t key = weight_key(w);
            if (j >= q.lo && j < q.hi && (D == 0 || key >> (kShift[D] + kWidth[D]) == border.least >> (kShift[D] + kWidth[D])))
                atomicAdd(&bins[first_bin(D) + (key >> kShift[D] & ((1u << kWidth[D]) - 1))], 1u);
        });
        __syncthreads();
        return next_digit<D>(border, want, bins);
    };
    if (want > 0 && count(std::integral_constant<int, 0>()) && count(std::integral_constant<int, 1>()))
        count(std::integral_constant<int, 2>());
    return border;
}

template <int T, int N>
__global__ __launch_bounds__(T) void k_select(EvictArgs a)
{
    __shared__ __align__(16) uint32_t bins[kBins];
    __shared__ uint64_t counts[N * (T / kWave)], sums[T / kWave];
    __shared__ int first_moved;
    const int sh = blockIdx.x, tid = threadIdx.x;
    const Kept q(a, sh / a.from.kv_heads);
    const float* w = a.from.weight + (int64_t)sh * a.from.weight_stride;
    float v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i * T + tid < q.L ? w[i * T + tid] : 0.0f;
    for (int b = tid; b < kBins; b += T) bins[b] = 0;
    if (tid == 0) first_moved = q.k;
    const Border border = find_border(q, bins, [&](auto&& f) {
#pragma unroll
        for (int i = 0; i < N; ++i) f(i * T + tid, v[i]);
    });
    __syncthreads();  // (every weight is in registers: in place, they may be overwritten)
    uint64_t done = 0;
    int moved = INT32_MAX;
    put_kept<T>(a, q, border, sh, 0, v, counts, sums, &done, &moved);
    finish<T>(a, q, sh, moved, &first_moved);
}

// In place, a pass's weights are all in registers before any is written, and go to places
// not past those already read.
__global__ __launch_bounds__(kSelLong) void k_select_long(EvictArgs a)
{
    constexpr int T = kSelLong, N = 16;
    __shared__ __align__(16) uint32_t bins[kBins];
    __shared__ uint64_t counts[N * (T / kWave)], sums[T / kWave];
    __shared__ int first_moved;
    const int sh = blockIdx.x, tid = threadIdx.x;
    const Kept q(a, sh / a.from.kv_heads);
    const float* w = a.from.weight + (int64_t)sh * a.from.weight_stride;
    for (int b = tid; b < kBins; b += T) bins[b] = 0;
    if (tid == 0) first_moved = q.k;
    const Border border = find_border(q, bins, [&](auto&& f) {
        constexpr int U = 16;  // loads in flight
        for (int j0 = 0; j0 < q.L; j0 += U * T) {
            float v[U];
#pragma unroll
            for (int i = 0; i < U; ++i) v[i] = j0 + i * T + tid < q.L ? w[j0 + i * T + tid] : 0.0f;
#pragma unroll
            for (int i = 0; i < U; ++i) f(j0 + i * T + tid, v[i]);
        }
    });
    uint64_t done = 0;
    int moved = INT32_MAX;
    for (int j0 = 0; j0 < q.L; j0 += N * T) {
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = j0 + i * T + tid < q.L ? w[j0 + i * T + tid] : 0.0f;
        __syncthreads();
        put_kept<T>(a, q, border, sh, j0, v, counts, sums, &done, &moved);
    }
    finish<T>(a, q, sh, moved, &first_moved);
}

// The kept tokens' keys and values to their places. A block takes chunks of whole places,
// up to kMoveUnits 16-byte pieces a thread, in turn; in place there is one block for each
// (sequence, kv head, K or V, column part), whose loads of a chunk are done before its stores
// begin: a kept token only ever moves down, so a later chunk reads nothing that an earlier
// one wrote. HBM bound into other pages: 256 heads of 2,048 tokens of up to 8,000 115-117 us for
// 546 MB, the rate of a large copy; in place, a chain of loads and stores in each block, 154.
constexpr int kMoveUnits = 4;  // 16-byte pieces of a thread in flight
__global__ __launch_bounds__(kBlock) void k_move(EvictArgs a)
{
    int id = blockIdx.x;
    const int block = id % a.blocks;
    id /= a.blocks;
    const int col = id % a.col_parts;
    id /= a.col_parts;
    const bool is_v = id & 1;
    const int sh = id >> 1, s = sh / a.from.kv_heads, h = sh - s * a.from.kv_heads;
    const EvictInfo info = a.info[sh];
    if (block == 0 && col == 0 && !is_v && h == 0 && threadIdx.x == 0) a.to.length[s] = info.kept;
    const int units = a.units.n;
    const uint8_t* src = (is_v ? a.from.v + h * a.from.v_head : a.from.k + h * a.from.k_head) + (int64_t)col * units * 16;
    uint8_t* dst = (is_v ? a.to.v + h * a.to.v_head : a.to.k + h * a.to.k_head) + (int64_t)col * units * 16;
    const int64_t sp = is_v ? a.from.v_page : a.from.k_page, st = is_v ? a.from.v_tok : a.from.k_tok;
    const int64_t dp = is_v ? a.to.v_page : a.to.k_page, dt = is_v ? a.to.v_tok : a.to.k_tok;
    const int smask = (1 << a.from.page_shift) - 1, dmask = (1 << a.to.page_shift) - 1;
    const int32_t* idx = a.kept_idx + (int64_t)sh * a.idx_stride;
    const Group& per = a.units;
    const int rows = kBlock * kMoveUnits / units;  // of a chunk
    for (int64_t r0 = info.first_moved + (int64_t)block * rows; r0 < info.kept; r0 += (int64_t)a.blocks * rows) {
        const int end = min(rows, info.kept - (int)r0) * units;
        u32x4 x[kMoveUnits];
#pragma unroll
        for (int i = 0; i < kMoveUnits; ++i) {
            const int p = i * kBlock + threadIdx.x, row = per.of(p), to = (int)r0 + row;
            x[i] = u32x4{0, 0, 0, 0};
            if (p < end) {
                const int j = idx[to];
                const int page = page_at(a.from, s, j >> a.from.page_shift);
                if (page >= 0) x[i] = *(const u32x4*)(src + page * sp + (j & smask) * st + (p - row * units) * 16);
            }
        }
        if (a.in_place) __syncthreads();
#pragma unroll
        for (int i = 0; i < kMoveUnits; ++i) {
            const int p = i * kBlock + threadIdx.x, row = per.of(p), to = (int)r0 + row;
            if (p < end) {
                const int page = page_at(a.to, s, to >> a.to.page_shift);
                if (page >= 0) *(u32x4*)(dst + page * dp + (to & dmask) * dt + (p - row * units) * 16) = x[i];
            }
        }
    }
}

template <typename K, typename A>
int enqueue(K kernel, int64_t blocks, int threads, void* stream, void* ev0, void* ev1, const A& a)
{
    if (blocks <= 0) return kNoLaunch;
    if (ev0 && ev1)
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, (hipStream_t)stream, (hipEvent_t)ev0,
                              (hipEvent_t)ev1, 0, a);
    else
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}

}  // namespace

void append_shape(AppendArgs& a)
{
    a.lanes = 1;
    while (a.lanes * 16 < a.c.dim) a.lanes *= 2;
    const int per = kWave / a.lanes, rounds = (a.heads + 2 * a.c.kv_heads + per - 1) / per;
    // few rows: a row's heads over several wavefronts
    const int most = (rounds + 3) / 4;
    a.parts = (int)std::max<int64_t>(1, std::min<int64_t>(most, 2048 / std::max(a.ch.n_rows, 1)));
}

void evict_shape(EvictArgs& a)
{
    const int units = a.from.dim * (a.dtype == kBF16 ? 2 : 4) / 16;
    const int64_t rows = std::min(capacity(a.from), capacity(a.to));
    a.col_parts = 1;
    a.blocks = 1;
    if (!a.in_place) {
        a.blocks = (int)std::max<int64_t>(1, (rows * units + kBlock * kMoveUnits - 1) / (kBlock * kMoveUnits));
        a.blocks = std::min(a.blocks, 64);
    } else {
        while (a.col_parts < 4 && units % (2 * a.col_parts) == 0) a.col_parts *= 2;
    }
    a.units = make_group(units / a.col_parts);
}

int launch_append(const AppendArgs& a, void* st, void* e0, void* e1)
{
    const int64_t blocks = ((int64_t)a.ch.n_rows * a.parts + kWaves - 1) / kWaves;
    return a.dtype == kBF16 ? enqueue(k_append<kBF16>, blocks, kBlock, st, e0, e1, a)
                            : enqueue(k_append<kF32>, blocks, kBlock, st, e0, e1, a);
}

int launch_select(const EvictArgs& a, void* st, void* e0, void* e1)
{
    const int64_t blocks = (int64_t)a.from.n_seqs * a.from.kv_heads, cap = capacity(a.from);
    if (cap <= 16 * 256) return enqueue(k_select<256, 16>, blocks, 256, st, e0, e1, a);
    if (cap <= 16 * 512) return enqueue(k_select<512, 16>, blocks, 512, st, e0, e1, a);
    if (cap <= 16 * 1024) return enqueue(k_select<1024, 16>, blocks, 1024, st, e0, e1, a);
    if (cap <= kSelTokens) return enqueue(k_select<1024, kSelItems>, blocks, 1024, st, e0, e1, a);
    return enqueue(k_select_long, blocks, kSelLong, st, e0, e1, a);
}

int launch_move(const EvictArgs& a, void* st, void* e0, void* e1)
{
    return enqueue(k_move, (int64_t)a.from.n_seqs * a.from.kv_heads * 2 * a.col_parts * a.blocks, kBlock, st, e0, e1, a);
}

}  // namespace msao
