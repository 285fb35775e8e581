// msao_attend.hip -- gfx950 (CDNA4) kernels for attention of a chunk of new tokens
// over a paged cache, and for the attention weight that each cached token receives.
//
// Rows of a (sequence, kv head) are its n new tokens times the `group` query heads
// that share the kv head: all of them read the same keys and values, so they fill the
// columns of the matrix instructions, and K and V are read once for up to 128 rows (64 of
// float32; half as many of heads above 128 channels). For bf16 each p is rounded to bf16 for the
// second product, by 2^-8 of it at most: float32 products take eight times as long, and two bf16 pieces of
// p twice. Errors of whole rows against 64 bits are 0.0017-0.0023 then, of which the result's
// own rounding is 0.0016-0.0017. Scores, sums, lse and weight are not rounded.
//
// k_attend (up to 16 rows of bf16; float32): a wavefront takes 32 tokens at a time, K and V
// straight from memory into registers in whole rows, and nothing through LDS:
//   S^T = K Q^T    A operand: lane (c, i) holds 16 bytes of token i's row
//   O^T = V^T P^T  S^T leaves lane (c, q) with tokens 4c..4c+3 of each 16, which is a
//                  B operand as it stands once the instruction's k index is read as
//                  those tokens; its A operand wants, of the same tokens, one channel a
//                  lane: lane (c, i) loads channels [i*E, i*E+E) (E = padded dim / 16)
//                  of tokens 4c..4c+3 and turns the block round with byte permutes.
// The queries lie in LDS, from where each wavefront takes them tile by tile: what the
// registers hold besides (K and V on their way, the output, the scores) then leaves two
// wavefronts on a SIMD, so that loads, exponents and products of different ones overlap.
// The wavefronts of a workgroup take tiles in turn (for more rows than one holds two of them
// take the same tile, each for its half of the rows; the second reads it from a cache) and
// join at the end through LDS; workgroups that share a row's tokens leave parts in the
// workspace, which k_combine joins. The running maximum is a reference that moves only
// when a score passes it by more than 2^kSlack, so most tiles need no reduction across
// lanes and no rescaling.
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

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x3 __attribute__((ext_vector_type(3)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;

constexpr int kWave = 64;
constexpr int kBlock = 256;
constexpr int kWaves = kBlock / kWave;
constexpr float kSlack = 8.0f;     // log2 units a score may pass the reference by
constexpr int kFar = 0x7FFFFF00;   // an offset past every buffer: the load gives zeros
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ rsrc_t rsrc(const void* base, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, bytes, 0x00020000);
}

__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p)
{
    const uint64_t v = (uint64_t)p;
    return (const uint8_t*)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}

// Wavefronts on a SIMD that the registers are divided among: heads of 256 take more than half.
constexpr int waves_per_simd(int dp) { return dp == 256 ? 1 : 2; }

template <int DT> struct Type;
template <> struct Type<kBF16> { static constexpr int kSize = 2; };
template <> struct Type<kF32> { static constexpr int kSize = 4; };

// 32-bit words that hold E values, loaded in pieces of 16, 12 or 8 bytes; AUX: cache policy.
constexpr int kOnce = 2;  // nontemporal: read once
template <int W, int AUX>
__device__ __forceinline__ void load_words(uint32_t (&w)[W], rsrc_t r, int off)
{
    static_assert(W == 2 || W == 3 || W == 6 || W % 4 == 0, "");
    if constexpr (W == 3) {
        const u32x3 v = __builtin_amdgcn_raw_buffer_load_b96(r, off, 0, AUX);
#pragma unroll
        for (int e = 0; e < 3; ++e) w[e] = v[e];
    } else if constexpr (W == 2 || W == 6) {
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
            const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(r, off + 8 * i, 0, AUX);
            w[2 * i] = v.x;
            w[2 * i + 1] = v.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, off + 16 * i, 0, AUX);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[4 * i + e] = v[e];
        }
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const f32x2 v = {a, b};
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf2));
}

// A channel's sum by the weights' sum l (inv = 1 / l). A row of no token, or of scores of -inf
// alone, has l 0 (the largest score's term is near 1 otherwise) and is 0, whatever its sum of
// values times 0 is: NaN where a value is not finite.
__device__ __forceinline__ float normed(float acc, float inv, float l) { return l == 0.0f ? 0.0f : acc * inv; }

// N values to 8- or 16-byte aligned memory (4 bytes for two of bf16).
template <int DT, int N>
__device__ __forceinline__ void store_values(uint8_t* dst, const float* v)
{
    if constexpr (DT == kBF16) {
        if constexpr (N == 4) *(u32x2*)dst = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        else *(uint32_t*)dst = pack_bf16(v[0], v[1]);
    } else {
        if constexpr (N == 4) *(f32x4*)dst = f32x4{v[0], v[1], v[2], v[3]};
        else *(f32x2*)dst = f32x2{v[0], v[1]};
    }
}

// Whether a 32-bit word of values holds an infinity or a NaN; and the word without them.
template <int DT>
__device__ __forceinline__ bool strange(uint32_t w)
{
    if constexpr (DT == kF32) return (w & 0x7F800000u) == 0x7F800000u;
    return (w & 0x7F800000u) == 0x7F800000u || (w & 0x7F80u) == 0x7F80u;
}
template <int DT>
__device__ __forceinline__ uint32_t without_strange(uint32_t w)
{
    if constexpr (DT == kF32) return strange<DT>(w) ? 0u : w;
    return ((w & 0x7F800000u) == 0x7F800000u ? 0u : w & 0xFFFF0000u) | ((w & 0x7F80u) == 0x7F80u ? 0u : w & 0xFFFFu);
}

// Sum over the 16 lanes of a row, in each of them.
__device__ __forceinline__ float row_sum(float v)
{
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xF, 0xF, false));  // turned by 8
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xF, 0xF, false));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x122, 0xF, 0xF, false));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x121, 0xF, 0xF, false));
    return v;
}

// Which (sequence, kv head, ...) a block of the flattened grid has.
struct Place {
    int seq, head, n_new, begin, length;
};
__device__ __forceinline__ Place place_of(const AttendArgs& a, int sh)
{
    Place p;
    p.seq = sh / a.c.kv_heads;
    p.head = sh - p.seq * a.c.kv_heads;
    const Rows r = seq_rows(a.ch, p.seq);
    p.begin = r.begin;
    p.n_new = r.n;
    p.length = seq_length(a.c, p.seq);
    return p;
}

// What a launch attends to: every token of a sequence (kAll); or in its first workgroups the tokens that a group of
// sequences shares, for the rows of all of them, and in the others a sequence's tokens behind those (kBoth).
enum : int { kAll = 0, kBoth = 1 };

// Whether the prefixes' groups are a list that ascends.
__device__ __forceinline__ bool ascending(const PrefixDev& pre)
{
    return __ballot(!groups_ascend(pre, threadIdx.x & (kWave - 1), kWave)) == 0;
}

// The group that sequence s would be in: the last one that begins at it or before it; none of a list that does not ascend.
__device__ __forceinline__ int group_at(const PrefixDev& pre, int s)
{
    int n = 0;
    bool ascend = true;
    const int lane = threadIdx.x & (kWave - 1);
    for (int g = 0; g < pre.n_groups; g += kWave) {
        const bool in = g + lane < pre.n_groups;
        const int at = pre.group[min(g + lane, pre.n_groups)], end = pre.group[min(g + lane + 1, pre.n_groups)];
        n += __popcll(__ballot(in && at <= s));
        ascend = ascend && __ballot(in && at > end) == 0;
    }
    return ascend ? uniform(n) - 1 : -1;
}

// A workgroup's place in its part of the launch.
struct Grid {
    bool shared;
    int block, row_tiles, splits, pairs;
};
template <int MODE>
__device__ __forceinline__ Grid grid_of(const AttendArgs& a)
{
    if (MODE == kBoth && (int)blockIdx.x < a.pre.blocks)
        return Grid{true, (int)blockIdx.x, a.pre.row_tiles, a.pre.splits, a.pre.n_groups * a.c.kv_heads};
    return Grid{false, (int)blockIdx.x - (MODE == kBoth ? a.pre.blocks : 0), a.row_tiles, a.splits, a.c.n_seqs * a.c.kv_heads};
}

// The tiles of rows that read a part of a prefix lie on one XCD, whose L2 then has the part for all of them: every
// eighth workgroup is on the same one.
__device__ __forceinline__ void shared_place(const Grid& grid, int& sh, int& split, int& tile)
{
    const int units = grid.pairs * grid.splits, eight = grid.block / (8 * grid.row_tiles), in = grid.block - eight * 8 * grid.row_tiles;
    const int width = min(8, units - 8 * eight), unit = 8 * eight + in % width;
    tile = in / width;
    sh = unit / grid.splits;
    split = unit - sh * grid.splits;
}

// What it computes: whose rows, how many, the first token, whether rows see different ones.
struct Work {
    Place p;
    int n_rows, from;
    bool causal;
};
template <int MODE>
__device__ __forceinline__ Work work_of(const AttendArgs& a, const Grid& grid, int sh)
{
    Work w;
    w.from = 0;
    if (MODE == kBoth && grid.shared) {
        const int g = sh / a.c.kv_heads;
        const GroupRows r = group_rows(a.pre, a.ch, g);
        w.p.seq = r.first;
        w.p.head = sh - g * a.c.kv_heads;
        w.p.begin = r.begin;
        w.p.n_new = r.first < a.pre.n_seqs ? r.n : 0;
        w.p.length = group_tokens(a.pre, capacity(a.c), g);
        w.n_rows = ascending(a.pre) && w.p.length > 0 ? min(w.p.n_new, a.pre.max_rows) * a.group.n : 0;
        w.causal = false;
        return w;
    }
    w.p = place_of(a, sh);
    w.n_rows = min(w.p.n_new, a.ch.max_new) * a.group.n;
    w.causal = a.causal;
    if (MODE == kBoth)
        w.from = prefix_of(a.pre, a.ch, capacity(a.c), w.p.seq, group_at(a.pre, w.p.seq), Rows{w.p.begin, w.p.n_new}, w.p.length, a.causal);
    return w;
}

// Part `split` of the `seen` tokens from `from` on: how many parts there are, whether one is all there is to a
// row, the part's tokens, its place in the workspace.
struct Part {
    bool there, alone;
    int lo, hi, at;
};
template <int MODE>
__device__ __forceinline__ Part part_of(const AttendArgs& a, const Grid& grid, int seen, int from, int split)
{
    Part t;
    if (MODE == kBoth && grid.shared) {
        t.there = split < parts_of(seen, a.pre.part_tokens);
        t.alone = false;
        t.lo = split * a.pre.part_tokens;
        t.hi = min(seen, t.lo + a.pre.part_tokens);
        t.at = split;
        return t;
    }
    const int parts = MODE == kBoth ? min(parts_of(seen - from, a.part_tokens), a.splits) : parts_of(seen, a.part_tokens);
    t.there = split < max(parts, 1);
    t.alone = parts <= 1 && from == 0;
    t.lo = from + split * a.part_tokens;
    // (of a call with prefixes the last part has what is more than the caller thought)
    t.hi = MODE == kBoth && split >= parts - 1 ? seen : min(seen, t.lo + a.part_tokens);
    t.at = (MODE == kBoth ? a.part_base : 0) + split;
    return t;
}

// Rows of the sequence that the call computes (max_new bounds the grid).
__device__ __forceinline__ int call_rows(const AttendArgs& a, const Place& p) { return min(p.n_new, a.ch.max_new) * a.group.n; }

// Pages of 64 half tiles (16 tokens) of a wavefront, one a lane: lane i has half i % NH of
// tile first + i / NH of those that turn `turn` of `step` takes (every step-th of NH halves).
template <int NH>
__device__ __forceinline__ int lane_pages(const CacheDev& c, int seq, int lo, int hi, int turn, int step, int first)
{
    const int lane = threadIdx.x & (kWave - 1);
    const int64_t tok = (int64_t)lo + 16 * NH * (turn + step * ((int64_t)first + lane / NH)) + 16 * (lane % NH);
    return tok < hi ? page_at(c, seq, (int)(tok >> c.page_shift)) : -1;
}

// A 16-token half tile: its buffers and how many of its tokens there are.
struct Half {
    rsrc_t r;
    u32x4 words;  // the same as four words
    int n;
};
__device__ __forceinline__ Half half_of(const uint8_t* base, int64_t page_bytes, int64_t tok_bytes, int row_bytes, int page,
                                        int tok, int hi, int mask)
{
    Half h;
    h.n = page < 0 ? 0 : clamp_int(hi - tok, 0, 16);
    h.n = uniform(h.n);
    const int64_t off = page < 0 ? 0 : (int64_t)page * page_bytes + (int64_t)(tok & mask) * tok_bytes;
    const uint8_t* at = uniform(base + off);
    const int bytes = uniform(h.n > 0 ? (h.n - 1) * (int)tok_bytes + row_bytes : 0);
    h.r = rsrc(at, bytes);
    h.words = u32x4{(uint32_t)(uint64_t)at, (uint32_t)((uint64_t)at >> 32) & 0xFFFFu, (uint32_t)bytes, 0x00020000u};
    return h;
}

// Rows of queries in LDS, a row a line of DP values and 16 bytes that spread the banks.
// As a B operand lane (c, i) takes row i, 16 bytes from (16 bytes) * (4 s + c) for step s.
template <int DT, int DP>
struct Queries {
    static constexpr int kLine = DP * Type<DT>::kSize + 16;
    static constexpr int kPieces = DP * Type<DT>::kSize / 16;  // of a row
    // Piece `piece` of the row: zeros past the last row and past the head's channels.
    __device__ static __forceinline__ u32x4 fetch(const AttendArgs& a, const Place& p, int row, int n_rows, int piece)
    {
        const int tok = a.group.of(row), head = p.head * a.group.n + (row - tok * a.group.n);
        const int off = 16 * piece;
        if (row >= n_rows || off >= a.c.dim * Type<DT>::kSize) return u32x4{0, 0, 0, 0};
        return *(const u32x4*)(a.q + (int64_t)(p.begin + tok) * a.q_stride + (int64_t)head * a.c.dim * Type<DT>::kSize + off);
    }
    // `rows` rows from r0 by the whole workgroup; the caller waits for it.
    __device__ static __forceinline__ void fill(uint8_t* lds, const AttendArgs& a, const Place& p, int r0, int rows, int n_rows)
    {
        for (int i = threadIdx.x; i < rows * kPieces; i += kBlock) {
            const int row = i / kPieces, piece = i - row * kPieces;
            *(u32x4*)(lds + row * kLine + 16 * piece) = fetch(a, p, r0 + row, n_rows, piece);
        }
    }
    // Operands of 16 rows from line `row`.
    u32x4 v[kPieces / 4];
    __device__ __forceinline__ void take(const uint8_t* lds, int row) { take_line(lds, row + (int)(threadIdx.x & 15)); }
    __device__ __forceinline__ void take_line(const uint8_t* lds, int line)
    {
        const int lane = threadIdx.x & (kWave - 1);
        const uint8_t* src = lds + line * kLine + 16 * (lane >> 4);
#pragma unroll
        for (int s = 0; s < kPieces / 4; ++s) v[s] = *(const u32x4*)(src + 64 * s);
    }
};

// Scores of 16 tokens (rows of the result: lane (c, q) tokens 4c + r) and 16 queries.
template <int DT, int DP>
__device__ __forceinline__ f32x4 scores(const u32x4 (&k)[DP * Type<DT>::kSize / 64], const Queries<DT, DP>& q)
{
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < DP * Type<DT>::kSize / 64; ++i) {
        if constexpr (DT == kBF16) {
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[i]), __builtin_bit_cast(bf16x8, q.v[i]),
                                                        s, 0, 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[i][e]), __uint_as_float(q.v[i][e]), s, 0, 0, 0);
        }
    }
    return s;
}

// Offsets of a lane's pieces of a row of K; channels past the head read as zeros.
template <int DT, int DP>
struct KeyOffsets {
    int off[DP * Type<DT>::kSize / 64];
    __device__ __forceinline__ KeyOffsets(int64_t tok_bytes, int row_bytes)
    {
        const int lane = threadIdx.x & (kWave - 1), i = lane & 15, c = lane >> 4;
#pragma unroll
        for (int s = 0; s < DP * Type<DT>::kSize / 64; ++s) {
            const int at = 64 * s + 16 * c;
            off[s] = at < row_bytes ? i * (int)tok_bytes + at : kFar;
        }
    }
};

template <int DT, int DP, int MT, int RW, int MODE>
__global__ __launch_bounds__(kBlock, waves_per_simd(DP)) void k_attend(AttendArgs a)
{
    constexpr int ES = Type<DT>::kSize;
    constexpr int KS = DP * ES / 64;   // pieces of a row of K a lane holds
    constexpr int E = DP / 16;         // channels of V a lane holds of a token
    constexpr int VW = E * ES / 4;     // as 32-bit words
    constexpr int S = E % 4 == 0 ? 4 : 2;  // channels of a store
    // halves of a tile; of float32 heads of 96 and more the registers hold one
    constexpr int NH = DT == kF32 && DP >= 96 ? 1 : 2, TT = 16 * NH;
    constexpr int LDP = DP + 4;        // floats between rows in LDS: spreads the banks
    constexpr int TW = kWaves / RW;    // wavefronts that take different tiles
    // values that no other wavefront reads need no cache (long rows of one token: 176 -> 165 us);
    // keys stay for the weight pass (a call with it over 383 MB of keys: 295 us with keys read once
    // too, 267 without)
    constexpr int kValuesOnce = RW == 1 ? kOnce : 0;
    constexpr int kQBytes = RW * MT * 16 * Queries<DT, DP>::kLine, kOBytes = kWaves * 16 * LDP * 4;
    __shared__ __align__(16) uint8_t lds[kQBytes > kOBytes ? kQBytes : kOBytes];
    __shared__ float lds_m[kWaves][MT * 16], lds_l[kWaves][MT * 16];
    float (*lds_o)[16][LDP] = (float (*)[16][LDP])lds;  // once the queries are used up

    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    const int i16 = lane & 15, c = lane >> 4, rw = wave % RW, tw = wave / RW;
    // neighbouring blocks lie on different XCDs: the parts of a pair start at a place of its own,
    // so that first parts, which every sequence has, are spread; last tiles, which see most, first
    const Grid grid = grid_of<MODE>(a);
    int sh, split, tile;
    if (MODE == kBoth && grid.shared) shared_place(grid, sh, split, tile);
    else {
        const int per_pair = grid.row_tiles * grid.splits;
        sh = grid.block / per_pair;
        const int j = (grid.block - sh * per_pair + sh) % per_pair;
        split = j / grid.row_tiles;
        tile = grid.row_tiles - 1 - (j - split * grid.row_tiles);
    }
    const Work work = work_of<MODE>(a, grid, sh);
    const Place& p = work.p;
    const bool causal = work.causal;
    const int n_rows = work.n_rows, r0 = tile * RW * MT * 16;
    if (r0 >= n_rows) return;
    const int r_end = min(r0 + RW * MT * 16, n_rows);
    const int seen = group_sees(p.length, p.n_new, a.group, r_end - 1, causal);
    const Part part = part_of<MODE>(a, grid, seen, work.from, split);
    if (!part.there) return;
    const int lo = part.lo, hi = part.hi;

    const int row_bytes = a.c.dim * ES, mask = (1 << a.c.page_shift) - 1;
    const uint8_t* kb = a.c.k + (int64_t)p.head * a.c.k_head;
    const uint8_t* vb = a.c.v + (int64_t)p.head * a.c.v_head;
    const KeyOffsets<DT, DP> ko(a.c.k_tok, row_bytes);
    int vo[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) vo[r] = i16 * E * ES < row_bytes ? (4 * c + r) * (int)a.c.v_tok + i16 * E * ES : kFar;

    Queries<DT, DP>::fill(lds, a, p, r0, RW * MT * 16, n_rows);
    const int line0 = rw * MT * 16;                                       // the wavefront's rows
    const int used = clamp_int((n_rows - r0 - line0 + 15) / 16, 0, MT);   // and how many sixteens of them there are
    int last[MT];  // the last token that the lane's row sees
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int row = r0 + line0 + 16 * m + i16;
        last[m] = causal ? p.length - p.n_new + a.group.of(row) : p.length - 1;
    }
    const int least = causal ? p.length - p.n_new + a.group.of(r0) : p.length - 1;  // of all rows

    f32x4 o[MT][E];
    float ref[MT], sum[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        ref[m] = -INFINITY;
        sum[m] = 0.0f;
#pragma unroll
        for (int t = 0; t < E; ++t) o[m][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    const int tiles = (hi - lo + TT - 1) / TT;
    const int mine = used > 0 && tiles > tw ? (tiles - tw + TW - 1) / TW : 0;
    u32x4 kf[NH][KS];
    uint32_t vf[NH][4][VW];
    int pages = lane_pages<NH>(a.c, p.seq, lo, hi, tw, TW, 0);
    int kn[NH], next_n[NH];
    auto load_k = [&](int it) {
        const int tok = lo + TT * (tw + TW * it);
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const int page = __builtin_amdgcn_readlane(pages, (NH * it + h) & 63);
            const Half f = half_of(kb, a.c.k_page, a.c.k_tok, row_bytes, page, tok + 16 * h, hi, mask);
            next_n[h] = f.n;
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[h][s] = __builtin_amdgcn_raw_buffer_load_b128(f.r, ko.off[s], 0, 0);
        }
    };
    auto load_v = [&](int it) {
        const int tok = lo + TT * (tw + TW * it);
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const int page = __builtin_amdgcn_readlane(pages, (NH * it + h) & 63);
            const Half f = half_of(vb, a.c.v_page, a.c.v_tok, row_bytes, page, tok + 16 * h, hi, mask);
#pragma unroll
            for (int r = 0; r < 4; ++r) load_words<VW, kValuesOnce>(vf[h][r], f.r, vo[r]);
        }
    };
    if (mine > 0) {
        load_k(0);
        load_v(0);
    }
    __syncthreads();
    bool left_out = false;
    for (int it = 0; it < mine; ++it) {
        const int tok = lo + TT * (tw + TW * it);
        const bool seen_whole = tok + TT <= hi && tok + TT - 1 <= least;  // all of it, by every row
        bool whole = seen_whole;
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            kn[h] = next_n[h];
            whole = whole && kn[h] == 16;
        }
        float x[MT][4 * NH];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (m >= used) break;
            Queries<DT, DP> q;
            q.take(lds, line0 + 16 * m);
#pragma unroll
            for (int h = 0; h < NH; ++h) {
                const f32x4 s = scores<DT, DP>(kf[h], q);
#pragma unroll
                for (int r = 0; r < 4; ++r) x[m][4 * h + r] = s[r] * a.scale;
            }
        }
        // (V of this tile is on its way: the lanes' pages may be the next ones)
        if (it + 1 < mine) {
            if (((it + 1) & (64 / NH - 1)) == 0) pages = lane_pages<NH>(a.c, p.seq, lo, hi, tw, TW, it + 1);
            load_k(it + 1);
        }
        if (!whole) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int h = 0; h < NH; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int j = 4 * c + r;
                        if (j >= kn[h] || tok + 16 * h + j > last[m]) x[m][4 * h + r] = -INFINITY;
                    }
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (m >= used) break;
            float most = x[m][0];
#pragma unroll
            for (int e = 1; e < 4 * NH; ++e) most = fmaxf(most, x[m][e]);
            if (__ballot(most > ref[m] + kSlack) != 0) {
                most = fmaxf(most, __shfl_xor(most, 16));
                most = fmaxf(most, __shfl_xor(most, 32));
                // (a row that its own scores do not move stays as it is, bit for bit)
                const float up = most > ref[m] + kSlack ? most : ref[m];
                // (ref -inf: the sums are 0 and stay 0)
                const float sc = ref[m] == up ? 1.0f : ref[m] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref[m] - up);
                ref[m] = up;
                sum[m] *= sc;
#pragma unroll
                for (int t = 0; t < E; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[m][t][r] *= sc;
            }
            const float base = ref[m] == -INFINITY ? 0.0f : ref[m];
#pragma unroll
            for (int e = 0; e < 4 * NH; ++e) {
#pragma clang fp contract(off)
                // (of a rounded score: 0 where that is the reference, however far it is)
                x[m][e] = __builtin_amdgcn_exp2f(x[m][e] - base);
                sum[m] += x[m][e];
            }
        }
        if (!seen_whole && causal) {
            // a value that some rows must not see is 0 times its weight there, and that is NaN
            // for one that is not finite: such values stay out of the product (see below)
            bool any = false;
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int w = 0; w < VW; ++w) any = any || strange<DT>(vf[h][r][w]);
            if (__ballot(any) != 0) {
                left_out = true;
#pragma unroll
                for (int h = 0; h < NH; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int w = 0; w < VW; ++w) vf[h][r][w] = without_strange<DT>(vf[h][r][w]);
            }
        }
        if constexpr (DT == kBF16) {
            u32x4 pb[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) pb[m][e] = pack_bf16(x[m][2 * e], x[m][2 * e + 1]);
#pragma unroll
            for (int t = 0; t < E; ++t) {
                const uint32_t sel = t & 1 ? 0x07060302u : 0x05040100u;
                u32x4 vt;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    vt[e] = __builtin_amdgcn_perm(vf[e / 2][2 * (e & 1) + 1][t / 2], vf[e / 2][2 * (e & 1)][t / 2], sel);
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    if (m < used)
                        o[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt),
                                                                          __builtin_bit_cast(bf16x8, pb[m]), o[m][t], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int t = 0; t < E; ++t)
#pragma unroll
                        for (int m = 0; m < MT; ++m)
                            if (m < used)
                                o[m][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[h][r][t]), x[m][4 * h + r],
                                                                               o[m][t], 0, 0, 0);
        }
        if (it + 1 < mine) load_v(it + 1);
    }

    if (left_out) {
        // the values left out, to the rows that see them: whatever the weight, it is above 0, and
        // the sum is infinite or NaN. From the first tile that some row does not see all of
#pragma unroll 1
        for (int it = max(0, (least + 1 - lo) / TT - tw) / TW; it < mine; ++it) {
            const int tok = lo + TT * (tw + TW * it);
            if (tok + TT <= hi && tok + TT - 1 <= least) continue;
#pragma unroll 1
            for (int t = tok; t < min(tok + TT, hi); ++t) {
                const int page = page_at(a.c, p.seq, t >> a.c.page_shift);
                if (page < 0) continue;
                const uint8_t* src = vb + (int64_t)page * a.c.v_page + (int64_t)(t & mask) * a.c.v_tok;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        const int at = (4 * c + r) * E * ES + 4 * w;
                        const uint32_t v = at < row_bytes ? *(const uint32_t*)(src + at) : 0u;
                        const uint32_t bad = v ^ without_strange<DT>(v);
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            if (t > last[m]) continue;
                            if constexpr (DT == kF32) {
                                o[m][w][r] += __uint_as_float(bad);
                            } else {
                                o[m][2 * w][r] += __uint_as_float(bad << 16);
                                o[m][2 * w + 1][r] += __uint_as_float(bad & 0xFFFF0000u);
                            }
                        }
                    }
            }
        }
    }

    // join the wavefronts: references and sums, then the outputs 16 rows at a time
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        sum[m] += __shfl_xor(sum[m], 16);
        sum[m] += __shfl_xor(sum[m], 32);
        if (c == 0) {
            lds_m[wave][16 * m + i16] = ref[m];
            lds_l[wave][16 * m + i16] = sum[m];
        }
    }
    const int orow = threadIdx.x >> 4, od = (threadIdx.x & 15) * E;  // row and first channel that this thread writes
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        __syncthreads();
        if (r0 + 16 * m >= n_rows) break;
        float most = -INFINITY;
#pragma unroll
        for (int w = 0; w < TW; ++w) most = fmaxf(most, lds_m[w * RW + rw][16 * m + i16]);
        const float sc = ref[m] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref[m] - most);
        // lane (c, q): channel (4c + r) E + t of tile t
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int t = 0; t < E; ++t) lds_o[wave][i16][(4 * c + r) * E + t] = o[m][t][r] * sc;
        __syncthreads();
#pragma unroll
        for (int g = 0; g < RW; ++g) {
            const int line = 16 * m + orow, row = r0 + g * MT * 16 + line;
            if (row >= n_rows || od >= a.c.dim) continue;
            float mm = -INFINITY, l = 0.0f, acc[E];
#pragma unroll
            for (int w = 0; w < TW; ++w) mm = fmaxf(mm, lds_m[w * RW + g][line]);
#pragma unroll
            for (int w = 0; w < TW; ++w) {
                // (a reference that never moved: the sum is 0, or NaN where a score was NaN, which moves none)
                const float mw = lds_m[w * RW + g][line], lw = lds_l[w * RW + g][line];
                l += mw == -INFINITY ? lw : lw * __builtin_amdgcn_exp2f(mw - mm);
            }
#pragma unroll
            for (int t = 0; t < E; ++t) {
                acc[t] = lds_o[g][orow][od + t];
#pragma unroll
                for (int w = 1; w < TW; ++w) acc[t] += lds_o[w * RW + g][orow][od + t];
            }
            const int tok = a.group.of(row), head = p.head * a.group.n + (row - tok * a.group.n);
            const int64_t at = (int64_t)(p.begin + tok) * a.heads + head;
            if (part.alone) {
                const float inv = 1.0f / l;
                uint8_t* dst = a.out + (int64_t)(p.begin + tok) * a.out_stride + ((int64_t)head * a.c.dim + od) * ES;
                // (the head's last channels may be part of what the thread has)
#pragma unroll
                for (int t = 0; t < E; t += S) {
                    if (od + t >= a.c.dim) break;
#pragma unroll
                    for (int e = 0; e < S; ++e) acc[t + e] = normed(acc[t + e], inv, l);
                    store_values<DT, S>(dst + ES * t, &acc[t]);
                }
                if (od == 0) {
                    const float z = l == 0.0f ? -INFINITY : mm + __builtin_amdgcn_logf(l);
                    if (a.lse) a.lse[at] = z * kLn2;
                    if (a.lse2) a.lse2[at] = z;
                }
            } else {
                const int64_t all = (int64_t)a.ch.n_rows * a.heads;
                float* po = a.part_o + (part.at * all + at) * a.c.dim + od;
#pragma unroll
                for (int t = 0; t < E; t += S)
                    if (od + t < a.c.dim) store_values<kF32, S>((uint8_t*)(po + t), &acc[t]);
                if (od == 0) *(f32x2*)(a.part_ml + 2 * (part.at * all + at)) = f32x2{mm, l};
            }
        }
    }
}

// Many rows, bf16 (wide drafts, chunks of prompts): K and V are read once for 64 MT rows; from some
// 100 rows on bound by the matrix cores, the reads of LDS and the exponents together: for heads of 128
// a workgroup reads 64 KB of LDS for 32 tokens, 512 clocks at 128 bytes, and its products take 515;
// for heads of 256, whose K and V serve 16 rows of a wavefront, 1,024 against 515. A stage of 64 tokens goes from memory to LDS without
// passing through registers (each wavefront brings 16 tokens) while the stage before it is
// used. Every wavefront has 16 MT rows of its own and takes all of the tokens, 32 at a time:
//   S^T = K Q^T with the queries in registers and K's rows as A operands,
//   O^T = V^T P^T with V's channels as A operands, by the reads that transpose 4 x 16 blocks
//   (lane (c, i): tokens 4c .. 4c+3 and 16+4c .. of channel i, the tokens of its P).
// In LDS the 16-byte pieces of a row are exchanged by a pattern of the row (K: piece ^ row,
// V: piece ^ 2 row), so that the lanes of a read, which lie in different rows, hit
// different banks; the lanes that bring a row choose their pieces accordingly.
typedef __attribute__((address_space(3))) uint8_t lds_byte;
typedef short s16x4 __attribute__((ext_vector_type(4)));

// 16 bytes a lane from `off` of a buffer straight to LDS, 1 KiB from the (uniform) address
// `to`; out of range zeros. As instructions of its own, because the compiler, which cannot
// tell the two stages apart, would wait for the next stage's loads before it reads this
// one's. The load has no register to write; it is waited for (stage_came) before the
// barrier after which its stage is read. The descriptor may have come from a vector instruction
// (readfirstlane), after which the hardware wants five wait states before a load reads it, and
// M0 one; the compiler counts none for text, so the text has six (attend_chunk 758 us, 753 with
// two). M0 is set for it alone: nothing else in the kernel uses M0.
// ONCE: the values of a call with one tile of rows need no cache, which keeps the keys for the
// weight pass (64 requests of 14 to 42 rows over up to 16,000 tokens: 146 us and 83 for the weight,
// 153 and 90 without; 8 such requests of 42 to 63 rows 29.8, 27.5 without).
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const u32x4& buffer, uint32_t to, int off)
{
    if constexpr (ONCE)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(to), "v"(off), "s"(buffer)
                     : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(buffer)
                     : "memory");
}
__device__ __forceinline__ void stage_came() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// A score s scale enters the exponent by one fused s scale - ref, which keeps what ref has lost of it by its rounding, up
// to 2^-24 of it: past 2^31 the power of that is infinite or 0 for the largest score itself. From kFarScore on a row's scale
// is the power of 2 below it, whose products are exact: its scores differ by 128 and more where they differ at all, and
// by half of that they have no weight as well. (A rounded product less ref would be an instruction more for each score.)
constexpr float kFarScore = 0x1p30f;
__device__ __forceinline__ bool is_far(float x) { return fabsf(x) >= kFarScore && fabsf(x) < INFINITY; }

constexpr int kRowLevel = 32;
template <int DP, int MT, int NW, int ST, int WPS, int MODE>
__global__ __launch_bounds__(NW * kWave, WPS) void k_attend_rows(AttendArgs a)
{
    constexpr int KS = DP / 32, VT = DP / 16;        // steps of a score; tiles of channels
    constexpr int CH = DP == 64 ? 8 : DP == 256 ? 32 : 16, RB = 16 * CH;  // 16-byte pieces of a row in LDS; its bytes
    constexpr int NI = 16 * CH / kWave;              // loads that bring 16 tokens
    __shared__ __align__(16) uint8_t lds_k[2][ST * RB], lds_v[2][ST * RB];
    __shared__ __align__(16) int lds_n[2][ST / 16];  // tokens that there are of each 16
    __shared__ int lds_left_out;

    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    const int i16 = lane & 15, c = lane >> 4;
    // the last tiles, which see most, of all pairs before the ones before them, so that no long
    // one is left to the end; a pair's kRowLevel tiles of a level side by side, which share keys
    // and values in the caches. 8 prompts of 1,500 tokens 71 us (83 pair by pair, 65 tile by tile),
    // one of 8,000 574 us (665, 543), chunks of 2,048 over 12,288 717 us (746, 780; the
    // clock takes 30 passes to rise, whose first take up to 1,020)
    const Grid grid = grid_of<MODE>(a);
    const int per_pair = grid.row_tiles * grid.splits, pairs = grid.pairs;
    int sh, split, tile;
    if (MODE == kBoth && grid.shared) shared_place(grid, sh, split, tile);
    else {
        const int level = min(grid.block / (kRowLevel * pairs), per_pair / kRowLevel), in_level = grid.block - level * kRowLevel * pairs;
        const int width = min(kRowLevel, per_pair - level * kRowLevel);
        sh = in_level / width;
        const int j = level * kRowLevel + (in_level - sh * width + sh) % width;
        split = j / grid.row_tiles;
        tile = grid.row_tiles - 1 - (j - split * grid.row_tiles);
    }
    const Work work = work_of<MODE>(a, grid, sh);
    const Place& p = work.p;
    const bool causal = work.causal;
    const int n_rows = work.n_rows, r0 = tile * NW * MT * 16;
    if (r0 >= n_rows) return;
    const int r_end = min(r0 + NW * MT * 16, n_rows);
    const int seen = group_sees(p.length, p.n_new, a.group, r_end - 1, causal);
    const Part part = part_of<MODE>(a, grid, seen, work.from, split);
    if (!part.there) return;
    const int lo = part.lo, hi = part.hi;

    const int row_bytes = a.c.dim * 2, mask = (1 << a.c.page_shift) - 1;
    const uint8_t* kb = a.c.k + (int64_t)p.head * a.c.k_head;
    const uint8_t* vb = a.c.v + (int64_t)p.head * a.c.v_head;
    constexpr int kTasks = ST / 8;  // 16 tokens of K or of V each
    int ko[NI], vo[NI];  // what a lane brings of 16 tokens
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int row = (n * kWave + lane) / CH, piece = lane % CH;
        const int kp = piece ^ (row & (CH - 1)), vp = piece ^ (2 * row & (CH - 1));
        ko[n] = 16 * kp < row_bytes ? row * (int)a.c.k_tok + 16 * kp : kFar;
        vo[n] = 16 * vp < row_bytes ? row * (int)a.c.v_tok + 16 * vp : kFar;
    }

    const int w0 = r0 + wave * MT * 16;                      // the wavefront's rows
    const int used = clamp_int((n_rows - w0 + 15) / 16, 0, MT);
    Queries<kBF16, DP> q[MT];
    int last[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int row = w0 + 16 * m + i16;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[m].v[s] = Queries<kBF16, DP>::fetch(a, p, row, n_rows, 4 * s + c) ^ (a.scale < 0.0f ? 0x80008000u : 0u);
        last[m] = causal ? p.length - p.n_new + a.group.of(row) : p.length - 1;
    }
    const int least = causal ? p.length - p.n_new + a.group.of(w0) : p.length - 1;
    const int least_of_all = causal ? p.length - p.n_new + a.group.of(r0) : p.length - 1;
    if (threadIdx.x == 0) lds_left_out = 0;
    // tokens that the wavefront's own last row sees
    const int w_hi = used > 0 ? min(hi, group_sees(p.length, p.n_new, a.group, min(w0 + MT * 16, n_rows) - 1, causal)) : lo;

    // the scale's sign is the queries', so that the largest product gives the largest score;
    // above 0, so that what is masked stays at -inf
    const float scale = fmaxf(fabsf(a.scale), 1.17549435e-38f);
    f32x4 o[MT][VT];
    float ref[MT], sum[MT], by[MT];  // by: the row's scale
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        by[m] = scale;
        ref[m] = -INFINITY;
        sum[m] = 0.0f;
#pragma unroll
        for (int t = 0; t < VT; ++t) o[m][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // where the lane's operands lie: K row i, pieces c ^ row + 4 s; V row 4c + i / 4, piece of
    // channels 4 (i % 4) .., half of it
    const int ka = i16 * RB + ((c ^ (i16 & (CH - 1))) << 4);
    const int vr = 4 * c + (i16 >> 2);
    const int va = vr * RB + ((((i16 & 3) >> 1) ^ (2 * vr & (CH - 1))) << 4) + 8 * (i16 & 1);

    const int stages = (hi - lo + ST - 1) / ST;
    static_assert(kTasks % NW == 0 || NW % kTasks == 0, "");
    const int half0 = wave % (ST / 16);  // the wavefront's 16 tokens of a stage, or the first of them
    int pages = 0;
    auto bring = [&](int st) {
        if ((st & 63) == 0) {
            const int64_t tok = (int64_t)lo + (int64_t)ST * (st + lane) + 16 * half0;
            pages = tok < hi ? page_at(a.c, p.seq, (int)(tok >> a.c.page_shift)) : -1;
        }
        const int tok = lo + ST * st + 16 * half0, page = __builtin_amdgcn_readlane(pages, st & 63);
        const bool does_k = NW < kTasks || wave < ST / 16, does_v = NW < kTasks || (wave >= ST / 16 && wave < kTasks);
        if (does_k) {
            const Half k = half_of(kb, a.c.k_page, a.c.k_tok, row_bytes, page, tok, hi, mask);
            lds_n[st & 1][half0] = k.n;
            const uint32_t to = uniform((int)(uint32_t)(uintptr_t)(lds_byte*)lds_k[st & 1]) + half0 * 16 * RB;
#pragma unroll
            for (int n = 0; n < NI; ++n) load_to_lds<false>(k.words, to + n * 1024, ko[n]);
        }
        if (does_v) {
            const Half v = half_of(vb, a.c.v_page, a.c.v_tok, row_bytes, page, tok, hi, mask);
            const uint32_t to = uniform((int)(uint32_t)(uintptr_t)(lds_byte*)lds_v[st & 1]) + half0 * 16 * RB;
#pragma unroll
            for (int n = 0; n < NI; ++n) load_to_lds<MT == 1 && DP != 256>(v.words, to + n * 1024, vo[n]);
        }
    };

    bool left_out = false;
    if (stages > 0) bring(0);
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): the queries, so that the loop need not wait for them
    for (int st = 0; st < stages; ++st) {
        // the stage has come, and nobody reads the other one any more
        stage_came();
        __syncthreads();
        if (st + 1 < stages) bring(st + 1);
        if (causal && !(lo + ST * st + ST <= hi && lo + ST * st + ST - 1 <= least_of_all)) {
            // some row does not see all of the stage: what is not finite of its values stays out of
            // the products (see k_attend). Each wavefront looks at the 16 tokens it brought
            if (NW < kTasks || (wave >= ST / 16 && wave < kTasks)) {
                uint8_t* mine = lds_v[st & 1] + half0 * 16 * RB + 16 * lane;
                bool any = false;
#pragma unroll
                for (int n = 0; n < NI; ++n) {
                    u32x4 w = *(const u32x4*)(mine + n * 1024);
                    const bool bad = strange<kBF16>(w[0]) || strange<kBF16>(w[1]) || strange<kBF16>(w[2]) || strange<kBF16>(w[3]);
                    any = any || bad;
                    if (bad) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = without_strange<kBF16>(w[e]);
                        *(u32x4*)(mine + n * 1024) = w;
                    }
                }
                if (any) lds_left_out = 1;
            }
            __syncthreads();
            left_out = uniform(lds_left_out) != 0;
        }
        int kn[ST / 16];
#pragma unroll
        for (int w = 0; w < ST / 16; ++w) kn[w] = uniform(lds_n[st & 1][w]);
        const uint8_t* sk = lds_k[st & 1];
        const uint8_t* sv = lds_v[st & 1];
#pragma unroll
        for (int u = 0; u < ST / kTile; ++u) {
            const int tok = lo + ST * st + kTile * u;
            if (tok >= w_hi) break;
            float x[MT][8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 kf[KS];
#pragma unroll
                for (int s = 0; s < KS; ++s) kf[s] = *(const u32x4*)(sk + (2 * u + h) * 16 * RB + (ka ^ s << 6));
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const f32x4 sc = scores<kBF16, DP>(kf, q[m]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[m][4 * h + r] = sc[r];
                }
            }
            const bool seen_whole = tok + kTile <= hi && tok + kTile - 1 <= least;
            if (!seen_whole || kn[2 * u] != 16 || kn[2 * u + 1] != 16) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int j = 4 * c + r;
                            if (j >= kn[2 * u + h] || tok + 16 * h + j > last[m]) x[m][4 * h + r] = -INFINITY;
                        }
            }
            u32x4 pb[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                float most = x[m][0];
#pragma unroll
                for (int e = 1; e < 8; ++e) most = fmaxf(most, x[m][e]);
                if (__ballot(most * by[m] > ref[m] + kSlack) != 0) {
                    most = fmaxf(most, __shfl_xor(most, 16));
                    most = fmaxf(most, __shfl_xor(most, 32));
                    const bool moves = most * by[m] > ref[m] + kSlack;
                    float up = moves ? most * by[m] : ref[m];
                    float sc = ref[m] == up ? 1.0f : ref[m] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref[m] - up);
                    if (__builtin_expect(__ballot(is_far(up) || by[m] != scale) != 0, 0) && moves) {
                        // (the old reference and the new one in the scale's own units, whichever they are in)
                        sc = __builtin_amdgcn_exp2f(fminf(ref[m] * (scale / by[m]) - most * scale, 0.0f));
                        by[m] = is_far(most * scale) ? __uint_as_float(__float_as_uint(scale) & 0x7F800000u) : scale;
                        up = most * by[m];
                    }
                    ref[m] = up;
                    sum[m] *= sc;
#pragma unroll
                    for (int t = 0; t < VT; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[m][t][r] *= sc;
                }
                const float base = ref[m] == -INFINITY ? 0.0f : ref[m];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[m][e] = __builtin_amdgcn_exp2f(fmaf(x[m][e], by[m], -base));
                    sum[m] += x[m][e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) pb[m][e] = pack_bf16(x[m][2 * e], x[m][2 * e + 1]);
            }
            auto value = [&](int t) {
                u32x4 w;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const lds_byte* at = (const lds_byte*)sv + (2 * u + h) * 16 * RB + (va ^ t << 5);
                    const u32x2 z = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at));
                    w[2 * h] = z.x;
                    w[2 * h + 1] = z.y;
                }
                return w;
            };
            auto add = [&](int t, const u32x4& w) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    o[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, pb[m]),
                                                                      o[m][t], 0, 0, 0);
            };
#pragma unroll
            for (int t = 0; t < VT; ++t) add(t, value(t));
        }
    }
    if (left_out) {
#pragma unroll 1
        for (int tok = lo + max(0, least_of_all + 1 - lo) / ST * ST; tok < w_hi; tok += ST) {
            if (tok + ST <= hi && tok + ST - 1 <= least_of_all) continue;
#pragma unroll 1
            for (int t = tok; t < min(tok + ST, hi); ++t) {
                const int page = page_at(a.c, p.seq, t >> a.c.page_shift);
                if (page < 0) continue;
                const uint8_t* src = vb + (int64_t)page * a.c.v_page + (int64_t)(t & mask) * a.c.v_tok;
#pragma unroll
                for (int v = 0; v < VT; ++v) {
                    const int at = (16 * v + 4 * c) * 2;
                    if (at >= row_bytes) continue;
                    const u32x2 w = *(const u32x2*)(src + at);
                    const uint32_t b0 = w.x ^ without_strange<kBF16>(w.x), b1 = w.y ^ without_strange<kBF16>(w.y);
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        if (t > last[m]) continue;
                        o[m][v][0] += __uint_as_float(b0 << 16);
                        o[m][v][1] += __uint_as_float(b0 & 0xFFFF0000u);
                        o[m][v][2] += __uint_as_float(b1 << 16);
                        o[m][v][3] += __uint_as_float(b1 & 0xFFFF0000u);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        sum[m] += __shfl_xor(sum[m], 16);
        sum[m] += __shfl_xor(sum[m], 32);
        if (by[m] != scale) ref[m] *= scale / by[m];  // (the quotient is exact)
        const int row = w0 + 16 * m + i16;
        if (row >= n_rows) continue;
        const int tok = a.group.of(row), head = p.head * a.group.n + (row - tok * a.group.n);
        const int64_t at = (int64_t)(p.begin + tok) * a.heads + head;
        if (part.alone) {
            const float inv = 1.0f / sum[m];
            auto of = [&](int t, int r) { return normed(o[m][t][r], inv, sum[m]); };
            uint8_t* dst = a.out + (int64_t)(p.begin + tok) * a.out_stride + (int64_t)head * row_bytes;
#pragma unroll
            for (int t = 0; t < VT; ++t) {
                const int ch = 16 * t + 4 * c;
                if (ch < a.c.dim)
                    *(u32x2*)(dst + 2 * ch) = u32x2{pack_bf16(of(t, 0), of(t, 1)), pack_bf16(of(t, 2), of(t, 3))};
            }
            if (c == 0) {
                const float z = sum[m] == 0.0f ? -INFINITY : ref[m] + __builtin_amdgcn_logf(sum[m]);
                if (a.lse) a.lse[at] = z * kLn2;
                if (a.lse2) a.lse2[at] = z;
            }
        } else {
            const int64_t all = (int64_t)a.ch.n_rows * a.heads;
            float* po = a.part_o + (part.at * all + at) * a.c.dim;
#pragma unroll
            for (int t = 0; t < VT; ++t)
                if (16 * t + 4 * c < a.c.dim) *(f32x4*)(po + 16 * t + 4 * c) = o[m][t];
            if (c == 0) *(f32x2*)(a.part_ml + 2 * (part.at * all + at)) = f32x2{ref[m], sum[m]};
        }
    }
}

// Parts of split rows joined: W wavefronts a row. DP / 4 lanes hold four channels each of a
// part; the lanes' groups take parts in turn, four in flight, and join at the end.
template <int DT, int DP, int W, int MODE>
__global__ __launch_bounds__(kBlock) void k_combine(AttendArgs a, int blocks_per)
{
    constexpr int ES = Type<DT>::kSize;
    constexpr int LP = DP == 96 ? 32 : DP / 4, kGroups = W * kWave / LP, kFly = 4;
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    const int sh = blockIdx.x / blocks_per;
    const Work work = work_of<MODE>(a, Grid{}, sh);
    const Place& p = work.p;
    const int from = work.from, n_rows = work.n_rows, row = (blockIdx.x - sh * blocks_per) * (kWaves / W) + wave / W;
    if (row >= n_rows) return;  // (W = kWaves: the whole block)
    const int r_end = min(row / a.tile_rows * a.tile_rows + a.tile_rows, n_rows);
    const int seen = group_sees(p.length, p.n_new, a.group, r_end - 1, a.causal);
    int shared = 0, parts = parts_of(seen, a.part_tokens);
    if constexpr (MODE == kBoth) {  // the prefix' parts, then the own ones, of which there is one at least
        shared = parts_of(from, a.pre.part_tokens);
        parts = min(parts_of(seen - from, a.part_tokens), a.splits);
        if (from > 0) parts = shared + max(parts, 1);
    }
    if (parts <= 1) return;  // written by k_attend
    const int tok = a.group.of(row), head = p.head * a.group.n + (row - tok * a.group.n);
    const int64_t all = (int64_t)a.ch.n_rows * a.heads, at = (int64_t)(p.begin + tok) * a.heads + head;
    const int t = wave % W * kWave + lane, group = t / LP, ch = (t & (LP - 1)) * 4;
    const bool has = ch < a.c.dim;
    float most = -INFINITY, l = 0.0f;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    auto join = [&](float m2, float l2, const f32x4& o2) {
        const float up = fmaxf(most, m2), base = up == -INFINITY ? 0.0f : up;
        const float s1 = __builtin_amdgcn_exp2f(most - base), s2 = __builtin_amdgcn_exp2f(m2 - base);
        most = up;
        l = l * s1 + l2 * s2;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = acc[e] * s1 + o2[e] * s2;
    };
    for (int i0 = group; i0 < parts; i0 += kGroups * kFly) {
        f32x2 ml[kFly];
        f32x4 o[kFly];
#pragma unroll
        for (int f = 0; f < kFly; ++f) {
            const int i = i0 + f * kGroups;
            ml[f] = f32x2{-INFINITY, 0.0f};
            o[f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (i < parts) {
                const int64_t j = MODE == kBoth && i >= shared ? a.part_base + i - shared : i;
                ml[f] = *(const f32x2*)(a.part_ml + 2 * (j * all + at));
                if (has) o[f] = *(const f32x4*)(a.part_o + (j * all + at) * a.c.dim + ch);
            }
        }
#pragma unroll
        for (int f = 0; f < kFly; ++f) join(ml[f].x, ml[f].y, o[f]);
    }
#pragma unroll
    for (int s = LP; s < kWave; s <<= 1) {
        f32x4 o2;
#pragma unroll
        for (int e = 0; e < 4; ++e) o2[e] = __shfl_xor(acc[e], s);
        join(__shfl_xor(most, s), __shfl_xor(l, s), o2);
    }
    if constexpr (W > 1) {
        __shared__ float lds[W][LP][6];
        if (lane < LP) {
            float* d = lds[wave][lane];
            d[0] = most;
            d[1] = l;
#pragma unroll
            for (int e = 0; e < 4; ++e) d[2 + e] = acc[e];
        }
        __syncthreads();
        if (threadIdx.x >= LP) return;
#pragma unroll
        for (int w = 1; w < W; ++w) {
            const float* d = lds[w][lane];
            join(d[0], d[1], f32x4{d[2], d[3], d[4], d[5]});
        }
    } else if (lane >= LP) return;
    const float inv = 1.0f / l;
    uint8_t* dst = a.out + (int64_t)(p.begin + tok) * a.out_stride + ((int64_t)head * a.c.dim + ch) * ES;
    if (has) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = normed(acc[e], inv, l);
        if constexpr (DT == kBF16) *(u32x2*)dst = u32x2{pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3])};
        else *(f32x4*)dst = acc;
    }
    if (ch == 0) {
        const float z = l == 0.0f ? -INFINITY : most + __builtin_amdgcn_logf(l);
        if (a.lse) a.lse[at] = z * kLn2;
        if (a.lse2) a.lse2[at] = z;
    }
}

constexpr float kMostSum = 0x1p24f;  // of a row that gives weight
__device__ __forceinline__ float weighing(float z) { return fabsf(z) >= kMostSum ? INFINITY : z; }

// The weight that each token receives, once the rows' sums (lse2) are known:
//   weight_j += sum_i 2^(x_ij - lse2_i).
// Lane (c, q) sums tokens 4c + r over its rows, and 16 lanes are added at the end. Every
// token has one wavefront, so no atomics, and the order of the sum is fixed.
// A row's sum is off by its rounding, 2^-24 of it, and so is the exponent: from 2^24 on nothing is known of x_ij - lse2_i,
// whose power is anything up to infinite past 2^31. Such rows add nothing, as ones that see nothing.
//
// Few rows (k_weight): K streams by, 16 tokens a wavefront, past the queries in LDS. HBM
// bound; 60 registers leave eight wavefronts on a SIMD, which is what hides the loads (32
// tokens in 94 registers: 100 us for attend_round's 383 MB against 91, which attention's nontemporal
// values made 83-89; two sets of registers in turn 112).
template <int DT, int DP, int MT>
__global__ __launch_bounds__(kBlock, waves_per_simd(DP)) void k_weight(AttendArgs a)
{
    constexpr int ES = Type<DT>::kSize;
    constexpr int KS = DP * ES / 64;
    __shared__ __align__(16) uint8_t lds[MT * 16 * Queries<DT, DP>::kLine];
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    const int i16 = lane & 15, c = lane >> 4;
    const int sh = blockIdx.x / a.weight_parts, part = (blockIdx.x - sh * a.weight_parts + sh) % a.weight_parts;
    const Place p = place_of(a, sh);
    const int n_rows = call_rows(a, p);
    if (n_rows == 0) return;
    const int seen = group_sees(p.length, p.n_new, a.group, n_rows - 1, a.causal);
    const int lo = part * a.weight_tokens, hi = min(seen, lo + a.weight_tokens);
    if (lo >= seen) return;
    const int row_bytes = a.c.dim * ES, mask = (1 << a.c.page_shift) - 1;
    const uint8_t* kb = a.c.k + (int64_t)p.head * a.c.k_head;
    const KeyOffsets<DT, DP> ko(a.c.k_tok, row_bytes);
    float* weight = a.c.weight + (int64_t)sh * a.c.weight_stride;
    Queries<DT, DP>::fill(lds, a, p, 0, MT * 16, n_rows);
    const int used = min((n_rows + 15) / 16, MT);
    // Columns behind the last row are that row again, with a sum of +inf, which gives 0 as for
    // rows of no weight: zeros for them would be NaN at an infinite key whose weight is 0
    float z[MT];
    int last[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int row = min(16 * m + i16, n_rows - 1), tok = a.group.of(row), head = p.head * a.group.n + (row - tok * a.group.n);
        z[m] = 16 * m + i16 < n_rows ? a.lse2[(int64_t)(p.begin + tok) * a.heads + head] : INFINITY;
        z[m] = weighing(z[m]);
        last[m] = a.causal ? p.length - p.n_new + tok : p.length - 1;
    }
    const int least = a.causal ? p.length - p.n_new : p.length - 1;
    const int tiles = (hi - lo + 15) / 16, mine = tiles > wave ? (tiles - wave + kWaves - 1) / kWaves : 0;
    u32x4 kf[KS];
    int n = 0, next_n = 0;
    int pages = lane_pages<1>(a.c, p.seq, lo, hi, wave, kWaves, 0);
    auto load_k = [&](int it) {
        const int page = __builtin_amdgcn_readlane(pages, it & 63);
        const Half f = half_of(kb, a.c.k_page, a.c.k_tok, row_bytes, page, lo + 16 * (wave + kWaves * it), hi, mask);
        next_n = f.n;
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[s] = __builtin_amdgcn_raw_buffer_load_b128(f.r, ko.off[s], 0, kOnce);
    };
    if (mine > 0) load_k(0);
    __syncthreads();
    for (int it = 0; it < mine; ++it) {
        const int tok = lo + 16 * (wave + kWaves * it) + 4 * c;  // the lane's first token
        n = next_n;
        const bool whole = n == 16 && tok - 4 * c + 15 <= least;
        float old[4], w[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int r = 0; r < 4; ++r) old[r] = i16 == 0 && 4 * c + r < n ? weight[tok + r] : 0.0f;
        auto add = [&](auto all_seen) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if (m >= used) break;
                Queries<DT, DP> q;
                q.take_line(lds, min(16 * m + i16, n_rows - 1));
                const f32x4 s = scores<DT, DP>(kf, q);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale, -z[m]));
                    if (decltype(all_seen)::value) w[r] += x;
                    else w[r] += 4 * c + r < n && tok + r <= last[m] ? x : 0.0f;
                }
            }
        };
        if (whole) add(std::true_type());
        else add(std::false_type());
        if (it + 1 < mine) {
            if (((it + 1) & 63) == 0) pages = lane_pages<1>(a.c, p.seq, lo, hi, wave, kWaves, it + 1);
            load_k(it + 1);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) w[r] = row_sum(w[r]);
        if (i16 == 0) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (4 * c + r < n) weight[tok + r] = old[r] + w[r];
        }
    }
}

// Many rows (k_weight_rows): a wavefront keeps the keys of 32 tokens, and the rows stream
// by through LDS, 64 at a time, the next ones on their way meanwhile. The rows that see a
// block's tokens are cut into row_parts parts, so that a few short prompts fill the
// device too; k_weight_join adds the parts' sums in order.
constexpr int kRowStep = 64;
constexpr int row_step(int dt, int dp) { return dt == kF32 && dp == 256 ? 16 : kRowStep; }  // registers
template <int DT, int DP>
__global__ __launch_bounds__(kBlock, waves_per_simd(DP)) void k_weight_rows(AttendArgs a)
{
    constexpr int ES = Type<DT>::kSize;
    constexpr int KS = DP * ES / 64, kStep = row_step(DT, DP);
    using Q = Queries<DT, DP>;
    constexpr int kPer = kStep * Q::kPieces / kBlock;  // pieces of a thread
    __shared__ __align__(16) uint8_t lds[kStep * Q::kLine];
    __shared__ float lds_z[kStep];
    __shared__ int lds_last[kStep];
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x >> 6);
    const int i16 = lane & 15, c = lane >> 4;
    const int per_pair = a.weight_parts * a.row_parts, sh = blockIdx.x / per_pair;
    const int j = (blockIdx.x - sh * per_pair + sh) % per_pair, block = j / a.row_parts, part = j - block * a.row_parts;
    const Place p = place_of(a, sh);
    const int n_rows = call_rows(a, p);
    const int seen = n_rows > 0 ? group_sees(p.length, p.n_new, a.group, n_rows - 1, a.causal) : 0;
    const int b0 = block * kTile * kWaves;
    if (b0 >= seen) return;
    const int tok = b0 + kTile * wave;
    const int row_bytes = a.c.dim * ES, mask = (1 << a.c.page_shift) - 1;
    const uint8_t* kb = a.c.k + (int64_t)p.head * a.c.k_head;
    const KeyOffsets<DT, DP> ko(a.c.k_tok, row_bytes);
    u32x4 kf[2][KS];
    int kn[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int t = tok + 16 * h, page = t < seen ? page_at(a.c, p.seq, t >> a.c.page_shift) : -1;
        const Half f = half_of(kb, a.c.k_page, a.c.k_tok, row_bytes, uniform(page), t, seen, mask);
        kn[h] = f.n;
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[h][s] = __builtin_amdgcn_raw_buffer_load_b128(f.r, ko.off[s], 0, 0);
    }
    // rows from the first that sees the block's first token, this part's share of them
    const int from = a.causal ? max(0, b0 - (p.length - p.n_new)) * a.group.n : 0;
    const int steps = (n_rows - from + kStep - 1) / kStep, per = (steps + a.row_parts - 1) / a.row_parts;
    const int s_end = min(steps, (part + 1) * per);
    float w[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    u32x4 next[kPer];
    float next_z = INFINITY;
    int next_last = -1;
    // Where a thread's pieces lie from the step's first token on. A group that divides the step
    // has each step start with a token's first head, and the offsets of all steps are one's
    uint32_t off[kPer];
    auto offsets = [&](int first_head) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int at = i * kBlock + threadIdx.x, line = at / Q::kPieces, row = first_head + line, t = a.group.of(row);
            off[i] = (uint32_t)t * (uint32_t)a.q_stride + (uint32_t)((row - t * a.group.n) * row_bytes + 16 * (at - line * Q::kPieces));
        }
    };
    const bool even = kStep % a.group.n == 0;
    if (even) offsets(0);
    auto fetch = [&](int step) {
        const int r0 = from + step * kStep, t0 = a.group.of(r0);
        const uint8_t* src = a.q + (int64_t)(p.begin + t0) * a.q_stride + (int64_t)p.head * a.group.n * row_bytes;
        if (!even) offsets(r0 - t0 * a.group.n);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int at = i * kBlock + threadIdx.x, line = at / Q::kPieces;
            next[i] = u32x4{0, 0, 0, 0};
            if (r0 + line < n_rows && 16 * (at - line * Q::kPieces) < row_bytes) next[i] = *(const u32x4*)(src + off[i]);
        }
        if (threadIdx.x < kStep) {
            const int row = r0 + threadIdx.x, t = a.group.of(row), head = p.head * a.group.n + (row - t * a.group.n);
            next_z = row < n_rows ? a.lse2[(int64_t)(p.begin + t) * a.heads + head] : INFINITY;
            next_z = weighing(next_z);
            next_last = row >= n_rows ? -1 : a.causal ? p.length - p.n_new + t : p.length - 1;
        }
    };
    if (part * per < s_end) fetch(part * per);
    for (int step = part * per; step < s_end; ++step) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int at = i * kBlock + threadIdx.x, row = at / Q::kPieces;
            *(u32x4*)(lds + row * Q::kLine + 16 * (at - row * Q::kPieces)) = next[i];
        }
        if (threadIdx.x < kStep) {
            lds_z[threadIdx.x] = next_z;
            lds_last[threadIdx.x] = next_last;
        }
        __syncthreads();
        if (step + 1 < s_end) fetch(step + 1);
        const int r0 = from + step * kStep;
        const int least = a.causal ? p.length - p.n_new + a.group.of(r0) : p.length - 1;
        const bool whole = kn[0] == 16 && kn[1] == 16 && tok + kTile - 1 <= least && r0 + kStep <= n_rows;
        auto add = [&](auto all_seen) {
#pragma unroll
            for (int m = 0; m < kStep / 16; ++m) {
                Q q;
                q.take(lds, 16 * m);
                const float z = lds_z[16 * m + i16];
                const int last = lds_last[16 * m + i16];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f32x4 s = scores<DT, DP>(kf[h], q);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int j = 4 * c + r;
                        const float x = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale, -z));
                        if (decltype(all_seen)::value) w[4 * h + r] += x;
                        else w[4 * h + r] += j < kn[h] && tok + 16 * h + j <= last ? x : 0.0f;
                    }
                }
            }
        };
        if (whole) add(std::true_type());
        else add(std::false_type());
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = row_sum(w[e]);
    if (i16 != 0) return;
    float* weight = a.c.weight + (int64_t)sh * a.c.weight_stride;
    float* mine = a.part_w + ((int64_t)part * a.c.n_seqs * a.c.kv_heads + sh) * capacity(a.c);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = tok + 16 * h + 4 * c + r;
            if (4 * c + r >= kn[h]) continue;
            if (a.row_parts == 1) weight[t] += w[4 * h + r];
            else mine[t] = w[4 * h + r];
        }
}

// Four tokens a thread (they share a page), eight parts in flight.
__global__ __launch_bounds__(kBlock) void k_weight_join(AttendArgs a, int blocks_per)
{
    const int sh = blockIdx.x / blocks_per;
    const Place p = place_of(a, sh);
    const int n_rows = call_rows(a, p);
    const int seen = n_rows > 0 ? group_sees(p.length, p.n_new, a.group, n_rows - 1, a.causal) : 0;
    const int t = ((blockIdx.x - sh * blocks_per) * kBlock + threadIdx.x) * 4;
    // (a token of no page got nothing)
    if (t >= seen || page_at(a.c, p.seq, t >> a.c.page_shift) < 0) return;
    const int64_t step = (int64_t)a.c.n_seqs * a.c.kv_heads * capacity(a.c);
    const float* src = a.part_w + (int64_t)sh * capacity(a.c) + t;
    f32x4 w = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i = 0; i < a.row_parts; i += 8) {
        f32x4 v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = i + e < a.row_parts ? *(const f32x4*)(src + (i + e) * step) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < 8; ++e) w += v[e];
    }
    float* dst = a.c.weight + (int64_t)sh * a.c.weight_stride + t;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (t + e < seen) dst[e] += w[e];
}

template <typename K, typename... A>
int enqueue(K kernel, int64_t blocks, void* stream, void* ev0, void* ev1, A... args)
{
    if (blocks <= 0) return kNoLaunch;
    if (ev0 && ev1)
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kBlock), 0, (hipStream_t)stream, (hipEvent_t)ev0,
                              (hipEvent_t)ev1, 0, args...);
    else
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kBlock), 0, (hipStream_t)stream, args...);
    return (int)hipGetLastError();
}

int padded_dim(int dim) { return dim <= 64 ? 64 : dim <= 96 ? 96 : dim <= 128 ? 128 : 256; }

int64_t pairs(const AttendArgs& a) { return (int64_t)a.c.n_seqs * a.c.kv_heads; }

// Of rows with many parts k_combine has the whole block on one row.
bool block_a_row(const AttendArgs& a) { return a.part_base + a.splits > 16; }

// bf16 rows go through k_attend_rows from 17 on: stages of 64 tokens serve all four wavefronts,
// where k_attend reads a tile once for each 32 rows (64 requests of up to 16,000 tokens: with 21
// to 28 rows 144 us, 151 through k_attend; 42 to 63 rows 153, 205; 70 to 126 rows 272, 461; one of
// 100,000 tokens with 126 rows 61, 91). Up to 16 rows k_attend (7 rows of 64 requests 134 us,
// 136 through the other; of 256 requests 185, 191; one row of two long ones 162, 164), but for
// heads of 256, of which its registers hold one wavefront a SIMD (two rows 135 us, 108 through
// the other). Up to 64 rows 16 rows a wavefront (42 to 63 rows: 162 us, with 32 and two
// wavefronts idle 168), beyond 32 a wavefront. Chunks of 2,048 over 12,288 tokens: 730 us, with
// 48 rows a wavefront 884 (246 registers, as fast a SIMD but fewer workgroups; 64 spill), 16
// rows and eight wavefronts 770, stages of 32 tokens 852 (each pair by pair; in levels 700-720).
// Heads of 256: 16 rows a wavefront and stages of 32, for the same registers and LDS (the
// same chunks 1.70 ms, 6.26 through k_attend). float32 stays with k_attend: the same chunks take
// 6.0 ms, 114 TFLOP/s of the 153 that a large product reaches (short ragged queries, which leave
// workgroups uneven and loads exposed, 39).
constexpr int kFewRows = 16;
constexpr int stage_of(int dp) { return dp == 256 ? 32 : 64; }
// Rows of a workgroup: what the registers of its wavefronts hold.
template <int DT, int DP, int MODE>
int attend_rows(const AttendArgs& a, void* st, void* e0, void* e1)
{
    const int64_t blocks = pairs(a) * attend_blocks(a).attend + (MODE == kBoth ? a.pre.blocks : 0);
    if constexpr (DT == kBF16) {
        constexpr int kPerSimd = DP == 64 ? 3 : 2;
        if (a.tile_rows == 64) return enqueue(k_attend_rows<DP, 1, kWaves, stage_of(DP), kPerSimd, MODE>, blocks, st, e0, e1, a);
        if constexpr (DP != 256) {
            if (a.tile_rows == 128) return enqueue(k_attend_rows<DP, 2, kWaves, stage_of(DP), kPerSimd, MODE>, blocks, st, e0, e1, a);
            if constexpr (MODE == kAll)
                if (a.tile_rows == 16) return enqueue(k_attend<DT, DP, 1, 1, MODE>, blocks, st, e0, e1, a);
        }
    } else {
        if (a.tile_rows == 16) return enqueue(k_attend<DT, DP, 1, 1, MODE>, blocks, st, e0, e1, a);
        if constexpr (DP == 256) {
            if (a.tile_rows == 32) return enqueue(k_attend<DT, DP, 1, 2, MODE>, blocks, st, e0, e1, a);
        } else {
            if (a.tile_rows == 32) return enqueue(k_attend<DT, DP, 2, 1, MODE>, blocks, st, e0, e1, a);
            if (a.tile_rows == 64) return enqueue(k_attend<DT, DP, 2, 2, MODE>, blocks, st, e0, e1, a);
        }
    }
    return (int)hipErrorInvalidValue;
}

template <int DT, int DP, int MODE>
int combine_rows(const AttendArgs& a, void* st, void* e0, void* e1)
{
    const int per = (int)attend_blocks(a).combine;
    return block_a_row(a) ? enqueue(k_combine<DT, DP, kWaves, MODE>, pairs(a) * per, st, e0, e1, a, per)
                          : enqueue(k_combine<DT, DP, 1, MODE>, pairs(a) * per, st, e0, e1, a, per);
}

template <int DT, int DP>
int weight_rows(const AttendArgs& a, void* st, void* e0, void* e1)
{
    const int64_t blocks = pairs(a) * attend_blocks(a).weight;
    const int64_t rows = (int64_t)a.ch.max_new * a.group.n;
    if (rows > kRowStep) return enqueue(k_weight_rows<DT, DP>, blocks, st, e0, e1, a);
    return rows <= 16 ? enqueue(k_weight<DT, DP, 1>, blocks, st, e0, e1, a) : enqueue(k_weight<DT, DP, 4>, blocks, st, e0, e1, a);
}

template <template <int, int> class F>
int by_type(const AttendArgs& a, void* st, void* e0, void* e1)
{
    const int dp = padded_dim(a.c.dim);
    if (a.dtype == kBF16)
        return dp == 64 ? F<kBF16, 64>::go(a, st, e0, e1) : dp == 96 ? F<kBF16, 96>::go(a, st, e0, e1)
             : dp == 128 ? F<kBF16, 128>::go(a, st, e0, e1) : F<kBF16, 256>::go(a, st, e0, e1);
    return dp == 64 ? F<kF32, 64>::go(a, st, e0, e1) : dp == 96 ? F<kF32, 96>::go(a, st, e0, e1)
         : dp == 128 ? F<kF32, 128>::go(a, st, e0, e1) : F<kF32, 256>::go(a, st, e0, e1);
}
template <int DT, int DP> struct Attend {
    static int go(const AttendArgs& a, void* st, void* e0, void* e1) { return attend_rows<DT, DP, kAll>(a, st, e0, e1); }
};
template <int DT, int DP> struct AttendShared {
    static int go(const AttendArgs& a, void* st, void* e0, void* e1) { return attend_rows<DT, DP, kBoth>(a, st, e0, e1); }
};
template <int DT, int DP> struct Combine {
    static int go(const AttendArgs& a, void* st, void* e0, void* e1) { return combine_rows<DT, DP, kAll>(a, st, e0, e1); }
};
template <int DT, int DP> struct CombineShared {
    static int go(const AttendArgs& a, void* st, void* e0, void* e1) { return combine_rows<DT, DP, kBoth>(a, st, e0, e1); }
};
template <int DT, int DP> struct Weight {
    static int go(const AttendArgs& a, void* st, void* e0, void* e1) { return weight_rows<DT, DP>(a, st, e0, e1); }
};

}  // namespace

// Parts of a row's tokens. Few rows: parts for kPartTarget workgroups if every sequence were
// as long as can be, of 128 .. 1,024 tokens (a tile a wavefront at least; 64 requests of up to
// 16,000 tokens with 14 to 42 rows: 153 us with the join for 1,024, 173 with 512, 161 with 2,048;
// two of 131,072 with one: 188 through a kernel of 166, 198, 186). More than 64 rows, whose
// parts cost a store and a load of 4 bytes a channel: none from 512 workgroups on (8 prompts of
// up to 1,500 tokens 79 us, 107 with parts of 256; 200 requests of up to 3,000 with 70 to 126 rows
// 240, 260 with parts of 1,024), below that parts for kManyTarget (8 requests of up to 16,000 with
// as many rows: 80 us), of at most 1,024 tokens where all rows are one workgroup's (64 requests: 346 us, 423
// with 4,000). float32, whose
// products take eight times as long, as many as for few rows (text over encoder states 70 us,
// 103 with parts for 512). Never parts for more than kMostParts workgroups: the workspace holds
// a part's output for each row of every sequence as if it were as long as the table allows, 3 to
// 50 GiB for 256 requests in tables of 2^17 to 2^20 tokens by parts of 1,024. (In a table of
// 2^17, against parts of 1,024: 256 requests of up to 3,000 tokens with 24 rows 457 us, 581; one of
// 100,000 among them 508, 628; 64 of up to 16,000 with 4 rows 224, 216, and with one of 120,000
// 296, 290; with 24 rows 313, 376.)
constexpr int64_t kPartTarget = 2048, kPartLeast = 128, kPartMost = 1024, kManyTarget = 1024, kManyTargetF32 = 4096, kMostParts = 16384;
// Parts of the tokens in the weight pass of few rows (attend_round 91 us, 93 with 8,192, before
// attention's values were nontemporal), and
// of the rows in that of many: up to 32 (25 us, 33 with 10).
constexpr int64_t kWeightTarget = 16384, kWeightLeast = 256, kWeightRowTarget = 8192, kMostRowParts = 32;
void attend_shape(AttendArgs& a)
{
    constexpr int64_t kMostGroups = (int64_t)1 << 30;  // more than a launch has; times a capacity below 2^60
    const int64_t rows = (int64_t)a.ch.max_new * a.group.n;
    const bool wide = padded_dim(a.c.dim) == 256;
    if (a.dtype == kBF16) a.tile_rows = rows <= kFewRows && !wide ? 16 : rows <= 64 || wide ? 64 : 128;
    else a.tile_rows = rows <= 16 ? 16 : rows <= 32 || wide ? 32 : 64;
    a.row_tiles = (int)((rows + a.tile_rows - 1) / a.tile_rows);
    const int64_t np = std::max<int64_t>(pairs(a), 1), groups = std::min(std::max<int64_t>(np * a.row_tiles, 1), kMostGroups), cap = capacity(a.c);
    auto up = [](int64_t v, int64_t to) { return (v + to - 1) / to * to; };
    const int64_t whole = std::max<int64_t>(up(cap, kTile), kTile);
    // parts for about kPartTarget workgroups if every sequence were as long as can be
    int64_t per = std::min<int64_t>(up((groups * cap + kPartTarget - 1) / kPartTarget, kPartLeast), kPartMost);
    if (rows > 64) {
        const int64_t target = a.dtype == kBF16 ? kManyTarget : kManyTargetF32;
        per = up((groups * cap + target - 1) / target, kPartLeast);
        if (a.row_tiles == 1) per = std::min(per, kPartMost);
        if (groups >= target / 2) per = whole;
    }
    per = std::max(per, up((groups * cap + kMostParts - 1) / kMostParts, kPartLeast));  // (a multiple of a stage)
    a.part_tokens = (int)std::min(std::max<int64_t>(per, kPartLeast), whole);
    a.splits = std::max(1, parts_of((int)cap, a.part_tokens));
    a.row_parts = 1;
    if (rows > kRowStep) {
        a.weight_tokens = kTile * kWaves;
        a.weight_parts = std::max(1, parts_of((int)cap, a.weight_tokens));
        const int64_t steps = (rows + kRowStep - 1) / kRowStep;
        a.row_parts = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(steps, kMostRowParts), kWeightRowTarget / (np * a.weight_parts)));
    } else {
        a.weight_tokens = (int)std::min<int64_t>(std::max<int64_t>(up((np * cap + kWeightTarget - 1) / kWeightTarget, kWeightLeast), kWeightLeast), whole);
        a.weight_parts = std::max(1, parts_of((int)cap, a.weight_tokens));
    }
}

// Of a call with shared prefixes. The prefixes' workgroups and the others are one launch, so that loads of the
// ones pass beside products of the others, and their tiles have the same rows, those of the prefixes (128 requests behind
// four documents of up to 16,384 tokens 142 us, in two launches 221, when that was chosen; 32 behind 6,016 tokens 28, 32). Parts
// for kSharedTarget workgroups if every group had the rows and tokens it can have (the 128 requests with the join 151 us
// for 1,024, 164 for 2,048, 190 for 4,096), of kSharedLeast tokens or more, as each writes and reads 512 bytes a row (the 32
// requests with the join 35 us for 256, 40 for 128, 32 for 512; small batches 9-10 for 256, 12-14 for 512), float32 of half as
// many (24 requests of float32 27 us with the join, 30). The other parts for kOwnTarget workgroups, by what sequences mostly
// have (the 128 requests 151 us, 142 for 1,024 and 137 for 4,096; the 32 requests 35, 39 and 35).
constexpr int64_t kSharedTarget = 1024, kSharedLeast = 256, kOwnTarget = 2048;
void shared_shape(AttendArgs& a, int max_own)
{
    const int page = 1 << a.c.page_shift;
    auto up = [](int64_t v, int64_t to) { return (v + to - 1) / to * to; };
    attend_shape(a);
    PrefixDev& pre = a.pre;
    const int64_t mine = (int64_t)a.ch.max_new * a.group.n, rows = std::max((int64_t)pre.max_rows * a.group.n, mine);
    const bool wide = padded_dim(a.c.dim) == 256;
    if (a.dtype == kBF16) a.tile_rows = rows <= 64 || wide ? 64 : 128;
    else a.tile_rows = rows <= 16 ? 16 : rows <= 32 || wide ? 32 : 64;
    a.row_tiles = (int)((mine + a.tile_rows - 1) / a.tile_rows);
    pre.row_tiles = (int)(((int64_t)pre.max_rows * a.group.n + a.tile_rows - 1) / a.tile_rows);
    const int64_t tiles = std::min<int64_t>((int64_t)pre.n_groups * a.c.kv_heads * pre.row_tiles, (int64_t)1 << 30);
    // (and of either no more than kMostParts tiles have: the workspace holds each part of every row)
    const int64_t all_tiles = ((int64_t)a.ch.n_rows * a.group.n + a.tile_rows - 1) / a.tile_rows * a.c.kv_heads;
    const int64_t least = a.dtype == kBF16 ? kSharedLeast : kSharedLeast / 2, most = pre.max_tokens;
    const int64_t per = std::max({least, (tiles * most + kSharedTarget - 1) / kSharedTarget, (all_tiles * most + kMostParts - 1) / kMostParts});
    pre.part_tokens = (int)std::min<int64_t>(up(per, kPartLeast), std::max<int64_t>(up(most, kPartLeast), kPartLeast));
    pre.splits = std::max(1, parts_of(pre.max_tokens, pre.part_tokens));
    a.part_base = pre.splits;
    const int64_t others = std::min<int64_t>(pairs(a) * a.row_tiles, (int64_t)1 << 30), cap = std::min<int64_t>(capacity(a.c), up(max_own, page));
    const int64_t mine_per = std::max(std::min<int64_t>((others * cap + kOwnTarget - 1) / kOwnTarget, kPartMost), (others * cap + kMostParts - 1) / kMostParts);
    a.part_tokens = (int)std::min<int64_t>(std::max<int64_t>(up(mine_per, kPartLeast), kPartLeast), std::max<int64_t>(up(cap, kTile), kTile));
    a.splits = std::max(1, parts_of((int)cap, a.part_tokens));
}

AttendBlocks attend_blocks(const AttendArgs& a)
{
    const int64_t rows = (int64_t)a.ch.max_new * a.group.n;
    AttendBlocks b{(int64_t)a.row_tiles * a.splits, 0, 0, 0};
    if (a.part_base + a.splits > 1) b.combine = block_a_row(a) ? rows : (rows + kWaves - 1) / kWaves;
    if (a.add_weight) b.weight = (int64_t)a.weight_parts * a.row_parts;
    if (a.add_weight && a.row_parts > 1) b.join = ((int64_t)capacity(a.c) + 4 * kBlock - 1) / (4 * kBlock);
    return b;
}

AttendBytes attend_bytes(const AttendArgs& a)
{
    const size_t rows = (size_t)a.ch.n_rows * (size_t)a.heads;
    AttendBytes b{0, 0, 0, 0};
    const size_t splits = (size_t)a.part_base + (size_t)a.splits;
    if (splits > 1) {
        b.part_o = rows * splits * (size_t)a.c.dim * 4;
        b.part_ml = rows * splits * 8;
    }
    if (a.add_weight) b.lse2 = rows * 4;
    if (a.add_weight && a.row_parts > 1) b.part_w = (size_t)a.row_parts * (size_t)pairs(a) * (size_t)capacity(a.c) * 4;
    return b;
}

int launch_attend(const AttendArgs& a, void* st, void* e0, void* e1) { return by_type<Attend>(a, st, e0, e1); }

int launch_shared(const AttendArgs& a, void* st, void* e0, void* e1) { return by_type<AttendShared>(a, st, e0, e1); }
int launch_shared_join(const AttendArgs& a, void* st, void* e0, void* e1) { return by_type<CombineShared>(a, st, e0, e1); }

int launch_combine(const AttendArgs& a, void* st, void* e0, void* e1)
{
    return a.splits <= 1 ? kNoLaunch : by_type<Combine>(a, st, e0, e1);
}

int launch_weight(const AttendArgs& a, void* st, void* e0, void* e1)
{
    return !a.add_weight ? kNoLaunch : by_type<Weight>(a, st, e0, e1);
}

int launch_weight_join(const AttendArgs& a, void* st, void* e0, void* e1)
{
    if (!a.add_weight || a.row_parts <= 1) return kNoLaunch;
    const int per = (int)attend_blocks(a).join;
    return enqueue(k_weight_join, pairs(a) * per, st, e0, e1, a, per);
}

}  // namespace msao
