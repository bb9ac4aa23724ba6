// The kernel of nkv_pages_prompt_attention for a prompt's chunk, instantiated a head dim at a time.
//
// With many columns the two products of 4 d operations a row and column are what it takes: they go through the matrix cores, 32 rows or dims x 32
// columns x 16 at a time, with
//   S = K Q^T     rows x columns, so that a lane holds 32 rows' logits of one column: maximum and sum in the lane, and one exchange with lane ^ 32
//   O^T = V^T P   dims x columns: the rows that a lane holds of S are those that the product takes from it as P, in that order; V's columns come from LDS
//                 transposed by the load (ds_read_b64_tr_b16)
// A workgroup takes kWaves x 32 columns of a unit, and walks over the pages that they see: a page is a tile of 64 rows, held twice in LDS, the next one on its way
// in registers (4-bit rows become 16-bit ones there, once for all columns).  K's products are exact; a weight is rounded to the rows' 16 bits, off by half
// a step of the type that the output is rounded to, and the sum that divides is that of the unrounded ones in fp32.  fp16 rows of 4-bit pages are outside of fp16's range
// where their scales are: they become bf16, exactly, and queries and weights are two pieces of bf16 then.
//
// What bounds it: 2048 tokens of 32 heads of 128 dims behind 30720 rows of 8 KV heads (1.07e12 operations) take 1040 to 1180 us, 0.9 to 1.0 PFLOP/s, by the card and how warm it is; a
// large matrix product reaches 1.27 on the same cards, and both are held back by power (zeros for inputs: 936 us, and 1.75 PFLOP/s).  The matrix cores are busy for 45 % of the cycles: a
// wavefront has six vector operations (exponentials, sums, roundings) for a product of 32 x 32 x 16, and a product holds up the SIMD's other wavefront's for 13 of its 32
// cycles.  LDS is active for 28 % of the cycles, without bank conflicts.  Tried: two groups of wavefronts that a barrier holds in opposite phases (products against
// exponentials): 1024 for 1046 us there, but 210 for 194 and 40 for 35 us in short prompts, where a page is seen by some wavefronts only; two pages between barriers
// (-2 %; at 192 dims +20); raised priority for the one or the other phase (no change).
#pragma once

#include "nkv_pages_prompt.h"

#include <algorithm>

namespace nkv {
namespace {

using f32x16 = float __attribute__((ext_vector_type(16)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));
using i16x4 = short __attribute__((ext_vector_type(4)));

template <int D, bool F16, bool FP4> struct Tile {
    static constexpr int kWaves = prompt_waves(D, F16 && FP4), kThreads = kWaves * 64, kCols = kWaves * 32;
    static constexpr bool kTwo = F16 && FP4;                              // two pieces
    static constexpr int kAtOnce = prompt_groups(D, kTwo) * kWaves / 4;    // wavefronts a SIMD
    static constexpr bool kHalf = F16 && !FP4;                            // the products' type is fp16
    static constexpr int kCpr = D / 8;                                    // 16-byte chunks of a row
    static constexpr int kStride = (D == 96 ? 128 : D) * 2;               // bytes of a row in LDS
    static constexpr int kMatrix = kRows * kStride;
    static constexpr int kItems = (kRows * kCpr + kThreads - 1) / kThreads;   // chunks a thread moves of K, and of V
    static constexpr bool kEven = kRows * kCpr % kThreads == 0;
    // fp16 weights of up to 2^(6 + 8), see kRoom: those of 2^-30 of the largest one still have all of their bits
    static constexpr float kShift = kHalf ? 6.f : 0.f;
};
enum Bends { kStraight, kSloped, kCapped };                                  // logits as they are, less slopes times distances, capped (with slopes or without)
constexpr int kProducts = 0x8, kReads = 0x100;   // groups of instructions, as sched_group_barrier numbers them
// A column's maximum is only moved when a logit is more than this above it (in powers of two): weights of up to 2^8 have the bits that those of up to 1 have, and
// the weighted values in their registers are seldom multiplied.
constexpr float kRoom = 8.f;

// Chunk c of a row lies at c ^ that.  LDS has 64 banks, 16 chunks: of K, any 16 rows that differ in their last four bits are in different banks; of V, the four rows by
// four chunks that 32 lanes transpose, and the eight rows by two chunks that lanes 0 .. 15 and 32 .. 47 do.
template <int STRIDE> __device__ __forceinline__ int k_swizzle(int row) { return STRIDE % 256 == 0 ? row & 15 : row >> 1 & 7; }
template <int STRIDE> __device__ __forceinline__ int v_swizzle(int row) { return STRIDE % 256 == 0 ? 4 * (row & 3) + (row >> 1 & 2) : 2 * (row & 2) + (row >> 1 & 2); }

template <bool HALF> __device__ __forceinline__ f32x16 product32(const u32x4 &a, const u32x4 &b, const f32x16 &c)
{
    if constexpr (HALF) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// V's rows that go to LDS: those behind the last one become zeros, since 0 times NaN is NaN.  Where some columns do not see all of the rows infinities and NaN become zeros as
// well, and their rows' bits are set in `odd`: the columns that do see them get a NaN for a logit.
template <bool HALF> __device__ __forceinline__ u32x4 only_finite(u32x4 y, int row, int valid, uint32_t *odd)
{
    constexpr uint32_t e = HALF ? 0x7c00u : 0x7f80u;
    bool found = false;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const bool lo = (y[w] & e) == e, hi = (y[w] >> 16 & e) == e;
        found |= lo || hi;
        y[w] = (lo ? 0u : y[w] & 0xffffu) | (hi ? 0u : y[w] & 0xffff0000u);
    }
    if (row >= valid) return u32x4{0u, 0u, 0u, 0u};
    if (found) atomicOr(odd + row / 32, 1u << row % 32);
    return y;
}

// A page on its way to LDS.  ODD: some columns do not see all of its rows, of which `valid` are there.
template <int D, bool F16, bool FP4> struct Stage {
    using T = Tile<D, F16, FP4>;
    uint32_t k[T::kItems][4], v[T::kItems][4];

    __device__ __forceinline__ void load(const uint8_t *__restrict__ page, int tid)
    {
        using P = WidePage<D>;
#pragma unroll
        for (int i = 0; i < T::kItems; ++i) {
            const int idx = i * T::kThreads + tid;
            if (!T::kEven && idx >= kRows * T::kCpr) break;
            const int row = idx / T::kCpr, c = idx - row * T::kCpr;
            const u32x4 x = *reinterpret_cast<const u32x4 *>(page + P::k(row, 8 * c)), y = *reinterpret_cast<const u32x4 *>(page + P::v(row, 8 * c));
#pragma unroll
            for (int w = 0; w < 4; ++w) k[i][w] = x[w], v[i][w] = y[w];
        }
    }
    template <bool ODD> __device__ __forceinline__ void store(uint8_t *lds_k, uint8_t *lds_v, int tid, int valid, uint32_t *odd) const
    {
#pragma unroll
        for (int i = 0; i < T::kItems; ++i) {
            const int idx = i * T::kThreads + tid;
            if (!T::kEven && idx >= kRows * T::kCpr) break;
            const int row = idx / T::kCpr, c = idx - row * T::kCpr;
            u32x4 y{v[i][0], v[i][1], v[i][2], v[i][3]};
            if constexpr (ODD) y = only_finite<T::kHalf>(y, row, valid, odd);
            *reinterpret_cast<u32x4 *>(lds_k + row * T::kStride + (c ^ k_swizzle<T::kStride>(row)) * 16) = u32x4{k[i][0], k[i][1], k[i][2], k[i][3]};
            *reinterpret_cast<u32x4 *>(lds_v + row * T::kStride + (c ^ v_swizzle<T::kStride>(row)) * 16) = y;
        }
    }
};

// 4 bits: pieces of 16 bytes, K's 2 D first, then V's; a wavefront's are all of one kind.  A piece of K is a block of a row, with its scale; of V four rows of 8 dims (of head dims from
// 192 on: two of 16), with the scales of four rows.  It becomes four chunks.  (A chunk at a time, 4 bytes and a scale each: 83 tokens of 64 heads of 256 dims over 320 units of 1531
// rows 382 us, so 237.)
template <int D, bool F16> struct Stage<D, F16, true> {
    using T = Tile<D, F16, true>;
    using P = Fp4Page<D>;
    static constexpr int kOf = 2 * D, kItems = (2 * kOf + T::kThreads - 1) / T::kThreads;
    u32x4 x[kItems];
    uint32_t scale[kItems];

    // V's piece: its quad of rows, the first of its rows in the quad, and its first chunk
    __device__ __forceinline__ static void place(int piece, int &quad, int &half, int &chunk)
    {
        if constexpr (P::C == 16) {
            half = 2 * (piece & 1);
            quad = piece / 2 / (D / 16);
            chunk = 2 * (piece / 2 - quad * (D / 16));
        } else {
            half = 0;
            quad = piece / (D / 8);
            chunk = piece - quad * (D / 8);
        }
    }
    __device__ __forceinline__ void load(const uint8_t *__restrict__ page, int tid)
    {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int piece = i * T::kThreads + tid;
            if (2 * kOf % T::kThreads != 0 && piece >= 2 * kOf) break;
            x[i] = *reinterpret_cast<const u32x4 *>(page + 16 * piece);
            if (piece < kOf) {
                scale[i] = page[P::k_scale(piece / P::NB, piece % P::NB)];
            } else {
                int quad, half, chunk;
                place(piece - kOf, quad, half, chunk);
                scale[i] = *reinterpret_cast<const uint32_t *>(page + P::v_scale(4 * quad, chunk / 4));
            }
        }
    }
    template <bool ODD> __device__ __forceinline__ void store(uint8_t *lds_k, uint8_t *lds_v, int tid, int valid, uint32_t *odd) const
    {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int piece = i * T::kThreads + tid;
            if (2 * kOf % T::kThreads != 0 && piece >= 2 * kOf) break;
            if (piece < kOf) {
                const int row = piece / P::NB, b = piece % P::NB;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<u32x4 *>(lds_k + row * T::kStride + ((4 * b + j) ^ k_swizzle<T::kStride>(row)) * 16) = codes(x[i][j], scale[i] << 23);
            } else {
                int quad, half, chunk;
                place(piece - kOf, quad, half, chunk);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int of_quad = P::C == 16 ? half + j / 2 : j, row = 4 * quad + of_quad, c = P::C == 16 ? chunk + j % 2 : chunk;
                    uint32_t w = x[i][j];
                    if constexpr (P::C == 4) w = (x[i][j / 2] >> 16 * (j % 2) & 0xffffu) | (x[i][2 + j / 2] >> 16 * (j % 2)) << 16;
                    u32x4 y = codes(w, (scale[i] >> 8 * of_quad & 255u) << 23);
                    if constexpr (ODD) y = only_finite<false>(y, row, valid, odd);
                    *reinterpret_cast<u32x4 *>(lds_v + row * T::kStride + (c ^ v_swizzle<T::kStride>(row)) * 16) = y;
                }
            }
        }
    }
    __device__ __forceinline__ static u32x4 codes(uint32_t w, uint32_t exponent)
    {
        const float s = __uint_as_float(exponent);
        return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3))};
    }
};

__device__ __forceinline__ float other_half(float x)                      // of lane ^ 32
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// grid: units * tiles * splits.  The unit changes first: a GPU's eight dies take workgroups in turn, so that a die works on few units at a time and finds their pages in its L2.  The
// last columns, which see the most rows, go first.
template <int D, bool F16, bool FP4, Bends BENT>
__global__ __launch_bounds__((Tile<D, F16, FP4>::kThreads), (Tile<D, F16, FP4>::kAtOnce)) void prompt_kernel(const PromptArgs a)
{
    using T = Tile<D, F16, FP4>;
    constexpr int kSteps = D / 16, kDims = D / 32;                        // of a row's products; of V's dims
    __shared__ __align__(16) uint8_t lds[2][2][T::kMatrix];
    __shared__ uint32_t odd[3][2];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, g = lane >> 5;
    int id = blockIdx.x;
    const int u = id % a.n_units;
    id /= a.n_units;
    const int split = id % a.splits, tile = a.tiles - 1 - id / a.splits;
    const int sq = u / a.H, h = u - sq * a.H, cols = a.n_new * a.G;
    const int len = rows_of(a.lens[u], a.max_pages), prefix = a.prefix ? max(0, min(a.prefix[sq], len)) : 0;
    const int32_t *table = a.table + (int64_t)u * a.max_pages;
    // rows that the workgroup's tokens, the wavefront's and the lane's stand on
    const int col_first = tile * T::kCols, col_last = min(cols, col_first + T::kCols) - 1;
    const int r_first = len - a.n_new + col_first / a.G, r_last = len - a.n_new + col_last / a.G;
    const int wcol = col_first + w * 32, wcol_last = min(cols - 1, wcol + 31);
    const bool works = wcol < cols;
    const int w_first = len - a.n_new + wcol / a.G, w_last = len - a.n_new + wcol_last / a.G;
    const int col = wcol + n;
    const bool there = col < cols;
    const int token = (there ? col : cols - 1) / a.G, head = (there ? col : cols - 1) - token * a.G, at = len - a.n_new + token;
    const int since = a.window > 0 ? max(at, 0) - a.window + 1 : 0;       // the first row of the lane's window
    const int64_t row_out = ((int64_t)sq * a.n_new + token) * a.H * a.G + h * a.G + head;

    const Seen seen = seen_pages(r_first, r_last, a.window, prefix);
    const int begin = (int)((int64_t)seen.count * split / a.splits), end = (int)((int64_t)seen.count * (split + 1) / a.splits);

    u32x4 q[T::kTwo ? 2 : 1][kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        u32x4 x = there && !a.flat ? *reinterpret_cast<const u32x4 *>(a.q + row_out * D + 16 * s + 8 * g) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] ^= a.flip;
        if constexpr (T::kTwo) {                                          // 11 bits: eight, and the three that are left
            float v[8], rest[8];
            unpack8<true>(x, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float cut = __uint_as_float(__float_as_uint(v[i]) & 0xffff0000u);
                rest[i] = v[i] - cut;
                v[i] = cut;
            }
            q[0][s] = pack8<false>(v);
            q[1][s] = pack8<false>(rest);
        } else {
            q[0][s] = x;
        }
    }
    float m = kNoMax, l = 0.f;
    f32x16 o[kDims];
#pragma unroll
    for (int t = 0; t < kDims; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    const float slope = BENT != kStraight && a.slopes ? a.slopes[h * a.G + head] * kToLog2 : 0.f;

    // the pages' numbers, 64 steps' at a time, one a lane: a load for every step would be waited for at every step
    int ids = -1;
    auto id_of = [&](int step) {
        if ((step - begin) % kWave == 0) ids = step + lane < end ? table[seen.page(step + lane)] : -1;
        return __builtin_amdgcn_readlane(ids, (step - begin) % kWave);
    };
    auto page_of = [&](int p) { return a.pool + (int64_t)(p >= 0 && p < a.n_pages ? p : 0) * (FP4 ? Fp4Page<D>::kBytes : WidePage<D>::kBytes); };
    // all rows of a page are seen by all tokens on rows r0 .. r1
    auto all_seen = [&](int first, int r0, int r1) { return r0 >= 0 && first + kRows <= len && (first + kRows <= prefix || (first + kRows - 1 <= r0 && (a.window <= 0 || first > r1 - a.window))); };
    auto none_seen = [&](int first, int r0, int r1) { return first >= prefix && (first > r1 || (a.window > 0 && first + kRows - 1 <= max(r0, 0) - a.window)); };

    Stage<D, F16, FP4> stage;
    int this_id = id_of(begin);
    auto put = [&](int step) {                                            // the staged page, of that step
        const int first = seen.page(step) * kRows, half = (step - begin) & 1;
        uint8_t *const lk = lds[half][0], *const lv = lds[half][1];
        if (all_seen(first, r_first, r_last)) stage.template store<false>(lk, lv, tid, kRows, nullptr);
        else stage.template store<true>(lk, lv, tid, len - first, odd[(step - begin) % 3]);
    };
    if (tid < 6) odd[tid / 2][tid % 2] = 0u;
    __syncthreads();
    if (begin < end) {
        stage.load(page_of(this_id), tid);
        put(begin);
    }
    __syncthreads();
    for (int step = begin; step < end; ++step) {
        const int first = seen.page(step) * kRows, half = (step - begin) & 1;
        const bool counts = this_id >= 0 && this_id < a.n_pages;
        this_id = id_of(step + 1);
        if (step + 1 < end) stage.load(page_of(this_id), tid);
        if (tid < 2) odd[(step - begin + 2) % 3][tid] = 0u;
        if (counts && works && !none_seen(first, w_first, w_last)) {
            const uint8_t *const lk = lds[half][0], *const lv = lds[half][1];
            // ---- S ----
            // Four steps' rows are asked for ahead of the products: a read from LDS takes as long as four of them.
            f32x16 s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
            constexpr int kAhead = kSteps < 4 ? kSteps : 4;
            u32x4 rows[kAhead][2];
            auto read_keys = [&](int k) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    rows[k % kAhead][t] = *reinterpret_cast<const u32x4 *>(lk + (32 * t + n) * T::kStride + ((2 * k + g) ^ k_swizzle<T::kStride>(n)) * 16);
            };
#pragma unroll
            for (int k = 0; k < kAhead; ++k) read_keys(k);
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if constexpr (T::kTwo) s[t] = product32<false>(rows[k % kAhead][t], q[1][k], s[t]);
                    s[t] = product32<T::kHalf>(rows[k % kAhead][t], q[0][k], s[t]);
                }
                if (k + kAhead < kSteps) read_keys(k + kAhead);
            }
            __builtin_amdgcn_sched_group_barrier(kReads, 2 * kAhead, 0);
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                __builtin_amdgcn_sched_group_barrier(kProducts, T::kTwo ? 4 : 2, 0);
                if (k + kAhead < kSteps) __builtin_amdgcn_sched_group_barrier(kReads, 2, 0);
            }
            float p[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) p[i] = s[i / 16][i % 16];
            const int base = first + 4 * g;                               // p[i] is of row base + row_at(i)
            auto row_at = [](int i) { return 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4; };
            // the page's rows that the lane's token sees, a bit each (in front of the unit's first row it sees nothing)
            const bool some = !all_seen(first, r_first, r_last);
            uint32_t sees[2] = {~0u, ~0u};
            if (some) {
                const int lo = max(since - first, 0), hi = at < 0 ? 0 : min(at + 1 - first, kRows), fr = at < 0 ? 0 : min(prefix - first, kRows);
                uint64_t bits = hi > lo ? ~0ull >> (kRows - (hi - lo)) << lo : 0ull;
                bits |= fr > 0 ? ~0ull >> (kRows - fr) : 0ull;
                sees[0] = (uint32_t)bits >> 4 * g, sees[1] = (uint32_t)(bits >> 32) >> 4 * g;
            }
            if constexpr (BENT == kCapped) {                             // (what a token does not see has no part in how the others are capped)
                float most = 0.f;
                if (some) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) most = fmaxf(most, __uint_as_float(__float_as_uint(p[i]) & (uint32_t)((int)(sees[i / 16] << (31 - row_at(i % 16))) >> 31) >> 1));
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) most = fmaxf(most, fabsf(p[i]));
                }
                bend(p, most, a.cap);
            }
            if (BENT == kSloped || (BENT == kCapped && a.slopes)) {
                const float from = (float)(at - base);
#pragma unroll
                for (int i = 0; i < 32; ++i) p[i] = fmaf(-slope, fabsf(from - (float)row_at(i)), BENT == kSloped ? p[i] * a.scale_log2 : p[i]);
            }
            if (some) {
                const uint64_t bad = (uint64_t)odd[(step - begin) % 3][1] << 32 | odd[(step - begin) % 3][0];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const uint32_t poison = (uint32_t)(bad >> 32 * t) >> 4 * g;
                    if (__any(poison != 0u)) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) p[16 * t + i] = poison & 1u << row_at(i) ? __uint_as_float(0x7fc00000u) : p[16 * t + i];
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) p[16 * t + i] = sees[t] & 1u << row_at(i) ? p[16 * t + i] : -INFINITY;
                }
            }
            // ---- weights ----
            const float scale = BENT != kStraight ? 1.f : a.scale_log2;
            float top = p[0];
#pragma unroll
            for (int i = 1; i < 32; ++i) top = fmaxf(top, p[i]);
            top = fmaxf(top, other_half(top)) * scale;
            if (__any(top > m + kRoom || fabsf(m) >= kFarMax)) {
                const float to = top > m + kRoom ? top : m, f = __builtin_amdgcn_exp2f(m - to);
                m = to;
                l *= f;
#pragma unroll
                for (int t = 0; t < kDims; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[t][i] *= f;
            }
            const bool far = fabsf(m) >= kFarMax && m > kNoMax;
            float factor = scale, less = T::kShift - m;
            if (__any(far)) {
#pragma clang fp contract(off)
#pragma unroll
                for (int i = 0; i < 32; ++i) p[i] = far ? p[i] * scale - m : p[i];
                if (far) factor = 1.f, less = T::kShift;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) p[i] = __builtin_amdgcn_exp2f(BENT != kStraight ? p[i] + less : fmaf(p[i], factor, less));
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 32; ++i) sum[i % 4] += p[i];
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            u32x4 wt[T::kTwo ? 2 : 1][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = p[8 * k + i];
                if constexpr (T::kTwo) {
                    float rest[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float cut = __uint_as_float(__float_as_uint(x[i]) & 0xffff0000u);
                        rest[i] = x[i] - cut;
                        x[i] = cut;
                    }
                    wt[1][k] = pack8<false>(rest);
                }
                wt[0][k] = pack8<T::kHalf>(x);
            }
            // ---- O ----
            constexpr int kMoves = 4 * kDims, kHeld = 4;
            u32x4 dims[kHeld];
            auto read_values = [&](int i) {
                const int k = i / kDims, t = i % kDims;
                const int vr = (lane & 15) / 4, vc = 2 * (lane >> 4 & 1) + (lane & 3) / 2, vb = 8 * (lane & 1);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint8_t *from = lv + (16 * k + 8 * j + 4 * g + vr) * T::kStride + ((4 * t + vc) ^ v_swizzle<T::kStride>(4 * g + vr)) * 16 + vb;
                    const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)from));
                    dims[i % kHeld][2 * j] = y.x, dims[i % kHeld][2 * j + 1] = y.y;
                }
            };
#pragma unroll
            for (int i = 0; i < kHeld; ++i) read_values(i);
#pragma unroll
            for (int i = 0; i < kMoves; ++i) {
                if constexpr (T::kTwo) o[i % kDims] = product32<false>(dims[i % kHeld], wt[1][i / kDims], o[i % kDims]);
                o[i % kDims] = product32<T::kHalf>(dims[i % kHeld], wt[0][i / kDims], o[i % kDims]);
                if (i + kHeld < kMoves) read_values(i + kHeld);
            }
            __builtin_amdgcn_sched_group_barrier(kReads, 2 * kHeld, 1);
#pragma unroll
            for (int i = 0; i < kMoves; ++i) {
                __builtin_amdgcn_sched_group_barrier(kProducts, T::kTwo ? 2 : 1, 1);
                if (i + kHeld < kMoves) __builtin_amdgcn_sched_group_barrier(kReads, 2, 1);
            }
        }
        if (step + 1 < end) put(step + 1);
        __syncthreads();
    }
    if (!there) return;
    l += other_half(l);
    if (a.splits > 1) {
        float *dst = a.part + (((int64_t)split * a.n_units + u) * cols + col) * (D + 4);
#pragma unroll
        for (int t = 0; t < kDims; ++t)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                *reinterpret_cast<f32x4 *>(dst + 32 * t + 8 * b + 4 * g) = f32x4{o[t][4 * b], o[t][4 * b + 1], o[t][4 * b + 2], o[t][4 * b + 3]};
        if (g == 0) dst[D] = m - T::kShift, dst[D + 1] = l;
        return;
    }
    const bool none = l == 0.f;                                           // (NaN is handed on)
    const float inv = none ? 0.f : 1.f / l;
#pragma unroll
    for (int t = 0; t < kDims; ++t)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            u32x2 y;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float x0 = none ? 0.f : o[t][4 * b + 2 * i] * inv, x1 = none ? 0.f : o[t][4 * b + 2 * i + 1] * inv;
                if constexpr (F16) y[i] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)x0, (_Float16)x1});
                else y[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x0, (__bf16)x1});
            }
            *reinterpret_cast<u32x2 *>(a.out + row_out * D + 32 * t + 8 * b + 4 * g) = y;
        }
    if (a.lse && g == 0) a.lse[row_out] = none ? -INFINITY : (m - T::kShift + log2f(l)) * kToLn;
}

// The splits' parts of a column: D / 4 threads, several columns a workgroup, eight parts asked for at once.  Bound by two trips to memory: 32 columns of 8 parts 3.4 us.
template <int D, bool F16> __global__ __launch_bounds__(256) void prompt_join_kernel(const PromptArgs a)
{
    constexpr int kLanes = D / 4, kAtOnce = 256 / kLanes;
    const int cols = a.n_new * a.G, e = threadIdx.x % kLanes * 4;
    const int64_t i = (int64_t)blockIdx.x * kAtOnce + threadIdx.x / kLanes, total = (int64_t)a.n_units * cols;
    if (threadIdx.x >= kLanes * kAtOnce || i >= total) return;
    float m = kNoMax, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    constexpr int kParts = 8;                                             // parts asked for at once
    for (int s0 = 0; s0 < a.splits; s0 += kParts) {
        f32x4 x[kParts];
        float pm[kParts], pl[kParts];
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            const float *p = a.part + (min(s0 + k, a.splits - 1) * total + i) * (D + 4);
            x[k] = *reinterpret_cast<const f32x4 *>(p + e);
            pm[k] = s0 + k < a.splits ? p[D] : kNoMax, pl[k] = p[D + 1];
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < kParts; ++k) top = fmaxf(top, pm[k]);
        const float f0 = __builtin_amdgcn_exp2f(m - top);
        m = top;
        l *= f0;
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] *= f0;
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            if (s0 + k >= a.splits) break;
            const float f = __builtin_amdgcn_exp2f(pm[k] - m);
            l = fmaf(f, pl[k], l);
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = fmaf(f, x[k][r], o[r]);
        }
    }
    const int u = (int)(i / cols), col = (int)(i - (int64_t)u * cols), sq = u / a.H, h = u - sq * a.H, token = col / a.G, head = col - token * a.G;
    const int64_t row = ((int64_t)sq * a.n_new + token) * a.H * a.G + h * a.G + head;
    const bool none = l == 0.f;
    u32x2 y;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const float x0 = none ? 0.f : o[2 * r] / l, x1 = none ? 0.f : o[2 * r + 1] / l;
        if constexpr (F16) y[r] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)x0, (_Float16)x1});
        else y[r] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x0, (__bf16)x1});
    }
    *reinterpret_cast<u32x2 *>(a.out + row * D + e) = y;
    if (a.lse && e == 0) a.lse[row] = none ? -INFINITY : (m + log2f(l)) * kToLn;
}

}  // namespace

template <int D> hipError_t launch_prompt_tiles(const PromptArgs &a, const nkv_pages &p, hipStream_t st)
{
    auto go = [&](auto f16, auto fp4) {
        constexpr bool F16 = decltype(f16)::value, FP4 = decltype(fp4)::value;
        const unsigned groups = (unsigned)((int64_t)a.n_units * a.tiles * a.splits);
        (a.cap.cap_log2 != 0.f ? prompt_kernel<D, F16, FP4, kCapped> : a.slopes ? prompt_kernel<D, F16, FP4, kSloped> : prompt_kernel<D, F16, FP4, kStraight>)<<<groups, Tile<D, F16, FP4>::kThreads, 0, st>>>(a);
        constexpr int kAtOnce = 256 / (D / 4);
        if (a.splits > 1) prompt_join_kernel<D, F16><<<(unsigned)(((int64_t)a.n_units * a.n_new * a.G + kAtOnce - 1) / kAtOnce), 256, 0, st>>>(a);
    };
    using Yes = std::true_type;
    using No = std::false_type;
    const bool f16 = p.dtype == NKV_DTYPE_F16, fp4 = p.format == NKV_PAGES_FP4;
    if (f16 && fp4) go(Yes{}, Yes{});
    else if (f16) go(Yes{}, No{});
    else if (fp4) go(No{}, Yes{});
    else go(No{}, No{});
    return hipGetLastError();
}

}  // namespace nkv
