// msao_pages.hip -- gfx950 (CDNA4) kernels that give the sequences of a paged cache the pages
// that their target lengths take, give back the ones they no longer need, and say where each
// new token lies.
//
// Sums over the sequences (pages taken, pages given back, rows) put every page and row in
// its place, so nothing is claimed by atomics and the same call gives the same tables. The
// i-th page taken, by sequence and column, is the i-th from the top of the stack of free
// pages, and the j-th given back becomes the j-th from its new top: a round's room that is
// given back is found again by the next round, and its stack is the one before it.
//
// Bound by latency: a few dependent loads. Up to 1,024 sequences and 8,192 rows one workgroup
// does everything in one launch, with its plans in LDS; beyond that it leaves them in the
// workspace, with a copy of the pages taken (the places they leave are given away meanwhile),
// and a second launch fills tables and slots from many workgroups.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "msao_cache.h"
#include "msao_internal.h"

namespace msao {
namespace {

constexpr int kWave = 64;
constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kFillThreads = 256;
constexpr int kAhead = 4;  // pages that a thread has on their way

struct Sums {
    int64_t take, back, rows;
};

// N values: the sums over the threads before this one in their place, and over all threads.
template <int N>
__device__ __forceinline__ void sum_before(int64_t (&v)[N], int64_t (&total)[N], int64_t (*room)[kWaves])
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
    auto scan = [&](int64_t x, int width) {
#pragma unroll
        for (int s = 1; s < width; s <<= 1) {
            const int64_t o = __shfl_up(x, s);
            if (lane >= s) x += o;
        }
        return x;
    };
    int64_t upto[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        upto[i] = scan(v[i], kWave);
        if (lane == kWave - 1) room[i][wave] = upto[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int64_t w = scan(lane < kWaves ? room[i][lane] : 0, kWaves);
        total[i] = __shfl(w, kWaves - 1);
        const int64_t b = __shfl(w, max(wave - 1, 0));
        v[i] = (wave > 0 ? b : 0) + upto[i] - v[i];
    }
    __syncthreads();
}

__device__ __forceinline__ int saturated(int64_t v) { return (int)(v < INT32_MAX ? v : INT32_MAX); }

// Plans of all sequences, their new lengths, columns, starts; what is taken and given back.
__device__ __forceinline__ Sums plan_all(const ResizeArgs& a, ResizePlan* plan, int64_t (*room)[kWaves], int count)
{
    Sums at{0, 0, 0};
    if (a.n_seqs == 0 && a.start && threadIdx.x == 0) a.start[0] = 0;
    int64_t taken = 0;  // by the sequences that get what they want
    for (int s0 = 0; s0 < a.n_seqs; s0 += kThreads) {
        const int s = s0 + threadIdx.x;
        const bool there = s < a.n_seqs;
        const int cap = a.per_seq << a.page_shift;
        int length = 0, want = 0, old = 0, need = 0;
        if (there) {
            length = clamp_int(a.length[s], 0, cap);
            want = clamp_int(a.want[s], 0, cap);
            const int held = a.held ? clamp_int(a.held[s], 0, a.per_seq) : 0;
            // (the held ones are named, whatever `columns` says: no page is taken in the place of one)
            old = a.columns ? max(clamp_int(a.columns[s], 0, a.per_seq), held) : columns_of(a, length, held);
            need = columns_of(a, want, held);
        }
        const int64_t asks = need > old ? need - old : 0;
        int64_t take[1] = {asks}, more[3], t_take[1], t_more[3];
        sum_before(take, t_take, room);
        take[0] += at.take;
        // (nobody behind one who gets no page takes any: what is left is not enough for its sum)
        const bool ok = asks == 0 || take[0] + asks <= count;
        if (!ok) {
            want = length;
            need = old;
        }
        const int64_t grows = want > length ? want - length : 0;
        more[0] = old > need ? old - need : 0;
        more[1] = grows;
        more[2] = ok ? asks : 0;
        sum_before(more, t_more, room);
        const int64_t row = at.rows + more[1];
        if (there) {
            plan[s] = ResizePlan{length, old, need, saturated(take[0]), (int)(at.back + more[0]), saturated(row)};
            a.length[s] = want;
            if (a.columns) a.columns[s] = need;
            if (a.start) {
                a.start[s] = saturated(row);
                if (s == a.n_seqs - 1) a.start[a.n_seqs] = saturated(row + grows);
            }
            if (a.granted) a.granted[s] = ok ? 1 : 0;
        }
        at = Sums{at.take + t_take[0], at.back + t_more[0], at.rows + t_more[1]};
        taken += t_more[2];
    }
    at.take = taken;
    return at;
}

// Pages taken into the tables, and the places of the new rows: items of `step` threads from `from` on.
// taken_at(i): the i-th page taken.
template <typename T>
__device__ __forceinline__ void fill(const ResizeArgs& a, const ResizePlan* plan, int64_t taken, int64_t rows, int from, int step, T taken_at)
{
    for (int64_t i = from; i < taken; i += step) {
        const int s = item_of(a.n_seqs, i, [&](int q) { return plan[q].take; });
        a.pages[(int64_t)s * a.table_stride + plan[s].columns + (int)(i - plan[s].take)] = taken_at(i);
    }
    if (rows > a.n_rows) rows = a.n_rows;
    for (int64_t r = from; r < rows; r += step) {
        const int s = item_of(a.n_seqs, r, [&](int q) { return plan[q].row; });
        const ResizePlan p = plan[s];
        const int pos = p.length + (int)(r - p.row), col = pos >> a.page_shift;
        if (a.positions) a.positions[r] = pos;
        if (!a.slots) continue;
        const int page = page_or_none(col < p.columns ? a.pages[(int64_t)s * a.table_stride + col] : taken_at(p.take + (col - p.columns)), a.n_pages);
        a.slots[r] = page < 0 ? -1 : ((int64_t)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
    }
}

// Pages given back, from the tables onto the stack; `base`: free pages below them.
__device__ __forceinline__ void give_back(const ResizeArgs& a, const ResizePlan* plan, int64_t back, int64_t base, int from, int step)
{
    if (back <= step) {  // few: each finds its sequence
        if (from >= back) return;
        const int s = item_of(a.n_seqs, from, [&](int q) { return plan[q].back; });
        int32_t* entry = a.pages + (int64_t)s * a.table_stride + plan[s].need + (from - plan[s].back);
        const int64_t to = base + back - 1 - from;
        if (to < a.n_pages) a.free[to] = *entry;  // (a stack of more pages than there are holds no more)
        *entry = -1;
        return;
    }
    // many: a wavefront has a sequence's, kAhead loads on their way (34,000 of 96 sequences by one workgroup 12 us, each found
    // by itself 31; of 4 sequences 21, 19; of one alone 61, 14, as the other wavefronts have none)
    const int lane = from & (kWave - 1);
    for (int s = from / kWave; s < a.n_seqs; s += step / kWave) {
        const ResizePlan p = plan[s];
        int32_t* entry = a.pages + (int64_t)s * a.table_stride + p.need;
        const int n = p.columns - p.need;
        const int64_t top = base + back - 1 - p.back;
        for (int c0 = lane; c0 < n; c0 += kAhead * kWave) {
            int32_t page[kAhead];
#pragma unroll
            for (int e = 0; e < kAhead; ++e) page[e] = c0 + e * kWave < n ? entry[c0 + e * kWave] : -1;
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                const int c = c0 + e * kWave;
                if (c >= n) break;
                if (top - c < a.n_pages) a.free[top - c] = page[e];
                entry[c] = -1;
            }
        }
    }
}

__global__ __launch_bounds__(kThreads) void k_resize_one(ResizeArgs a)
{
    __shared__ ResizePlan plan[kResizeSeqs];
    __shared__ int64_t room[3][kWaves];
    const int count = clamp_int(a.count[0], 0, a.n_pages);
    const Sums all = plan_all(a, plan, room, count);
    __syncthreads();
    fill(a, plan, all.take, all.rows, threadIdx.x, kThreads, [&](int64_t i) { return a.free[count - 1 - i]; });
    __syncthreads();  // the places of the pages taken may be given away
    give_back(a, plan, all.back, count - all.take, threadIdx.x, kThreads);
    if (threadIdx.x == 0) a.count[0] = (int)min(count - all.take + all.back, (int64_t)a.n_pages);
}

__global__ __launch_bounds__(kThreads) void k_resize_plan(ResizeArgs a)
{
    __shared__ int64_t room[3][kWaves];
    const int count = clamp_int(a.count[0], 0, a.n_pages);
    const Sums all = plan_all(a, a.plan, room, count);
    // (eight loads in flight: one by one 34,000 pages take 30 us)
    for (int64_t i0 = threadIdx.x; i0 < all.take; i0 += 8 * kThreads) {
        int32_t page[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) page[e] = i0 + e * kThreads < all.take ? a.free[count - 1 - i0 - e * kThreads] : 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i0 + e * kThreads < all.take) a.taken[i0 + e * kThreads] = page[e];
    }
    __syncthreads();  // every thread has read the count
    if (threadIdx.x == 0) {
        a.count[0] = (int)min(count - all.take + all.back, (int64_t)a.n_pages);
        a.moved[0] = (int)all.take;
        a.moved[1] = saturated(all.back);
        a.moved[2] = (int)(count - all.take);
        a.moved[3] = saturated(all.rows);
    }
}

__global__ __launch_bounds__(kFillThreads) void k_resize_fill(ResizeArgs a)
{
    const int from = blockIdx.x * kFillThreads + threadIdx.x, step = gridDim.x * kFillThreads;
    const int taken = a.moved[0], back = a.moved[1], base = a.moved[2], rows = a.moved[3];
    fill(a, a.plan, taken, rows, from, step, [&](int64_t i) { return a.taken[i]; });
    give_back(a, a.plan, back, base, from, step);
}

template <typename K>
int enqueue(K kernel, int64_t blocks, int threads, void* stream, void* ev0, void* ev1, const ResizeArgs& a)
{
    if (blocks <= 0) return kNoLaunch;
    if (ev0 && ev1)
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, (hipStream_t)stream, (hipEvent_t)ev0, (hipEvent_t)ev1, 0, a);
    else
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}

}  // namespace

int launch_resize(const ResizeArgs& a, void* st, void* e0, void* e1)
{
    return resize_in_one(a) ? enqueue(k_resize_one, 1, kThreads, st, e0, e1, a) : enqueue(k_resize_plan, 1, kThreads, st, e0, e1, a);
}

int launch_resize_fill(const ResizeArgs& a, void* st, void* e0, void* e1)
{
    if (resize_in_one(a)) return kNoLaunch;
    const int64_t items = std::max<int64_t>(a.n_rows, 8 * (int64_t)a.n_seqs);
    return enqueue(k_resize_fill, std::min<int64_t>((items + kFillThreads - 1) / kFillThreads, 4096), kFillThreads, st, e0, e1, a);
}

}  // namespace msao
