// What attention of few columns over pages is made of, for nkv_pages_attention and, with rules for the logits (RULES), nkv_pages_prompt_attention.
//
// For unit u and its columns (token, query head): s_i = scale <q, k_i>, out = sum_i softmax(s)_i v_i over the rows that the column sees.
// Every row is read once for up to 16 columns and used for 4 d multiply-adds a column: bound by memory, if the rest keeps up.
// Both products go through the matrix cores, exactly but for fp16 weights:
//   S = K Q^T     4-bit values become bf16, which holds them exactly (an fp16 query then in two bf16 pieces); 16 x 16 x 32 products
//                 over a lane's dims in turn.  (The scaled product of 4-bit rows as they lie in the page and 8-bit pieces of a query
//                 loses bits of small terms beside large ones: up to 6e-6 of the terms' sum, 2e-7 in the mean.)
//   O^T = V^T P   a weight is split into three bf16 pieces, which hold its 24 bits; for 16-bit rows of fp16 into two of fp16, which hold 22: off by 2^-22 of
//                 the weight at most, 1.4e-8 of an output over some thousand rows, where the sums in fp32 leave 2e-7.
// A column's running maximum, sum and weighted values stay in registers; with rows as the operands' other axis no lane
// exchange is needed between the products: the rows that a lane holds of S are those it holds of P, and V's rows are taken in that order.
//
// The pages of all units are cut into stretches of the same length, one for every wavefront that the device holds, whichever units they belong to: the lengths
// are on the device, so every wavefront finds its own by counting.  A stretch's part of a unit goes to the workspace as (maximum, sum, weighted
// values), that of a workgroup's four stretches in one unit as one, and pages_combine_kernel joins a unit's.  A wavefront works on 32 rows, half a page,
// while the next ones are on their way.
//
// Whole calls, us, and what reading the same bytes alone takes (6.8 TB/s): 36 x 8 units of about 8192 rows, head dim 128, 4 query heads a KV head, bf16, 4
// bits 65 (kernel 60.1), 49; one layer of them 10.1, 1.4: the launches, and three trips to memory one after the other (lengths, page, rows).  A call that
// fills the device takes some 10 us beside 4.1 a page and wavefront (6.5 TB/s); the vector and matrix instructions of that page take 2.8.
//
// RULES: the pages that a unit's tokens see are its prefix's and its windows', numbered through (seen_pages), so that stretches hold no page that nobody sees; logits are capped and
// lessened by distances in between; the output is rounded to 16 bits, so that a weight is rounded to them too, one product with V for three.  A decode step of 32 sequences, 8 KV
// heads of 8 query heads, 4100 of 8193 4-bit rows seen, capped: 38.4 us and 4.7 for the parts; its bytes alone 19.6.
// ALONE: a workgroup of eight wavefronts a unit, with nothing to count at the start and nothing to join at the end: 34.6 us there, in one launch.
#pragma once

#include "nkv_pages_prompt.h"

#include <algorithm>

namespace nkv {
namespace {

using f32x4 = float __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256, kWaves = kThreads / 64;
// Workgroups that a compute unit holds at once, by the registers that a head dim takes, and no more than that are launched.
__host__ __device__ constexpr int groups_at_once(int D) { return D == 64 ? 4 : D <= 128 ? 3 : 2; }
constexpr float kNone = -3.0e38f;        // running maximum before any row was seen
// A column's maximum is a rounded product with the scale, and its rows' logits are not rounded before they are taken from it: all of its weights are 2^(half of the
// maximum's last place) off at most, which their sum takes out again.  From here on that place is 2 or more, and weights could leave their type's range: logits are rounded
// alike, so that the largest weight is 1.
constexpr float kFar = 0x1p24f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ int clamp_len(int len, int max_pages) { return max(0, min(len, max_pages * kRows)); }

struct Parts;

struct AttendArgs {
    const uint16_t *q;
    const uint8_t *pool;
    const int32_t *table, *lens;
    int32_t n_units, H, G, n_new, n_pages, max_pages;
    float scale_log2;                    // positive, subnormal or not: rows that are not seen have the product -inf
    uint32_t flip;                       // sign bits of the query that change
    bool flat;                           // a scale of zero (in 32 bits): the query counts as zeros
    Parts *plan;                         // per unit
    float *part;                         // [part][column][D + 4]: weighted values, maximum, sum
    // RULES
    bool bent;                           // cap or slopes
    Cap cap;
    int32_t window;
    const float *slopes;
    const int32_t *prefix;
    // a workgroup a unit
    void *out;
    float *lse;
};

// COLS: columns a workgroup takes, 16, or of 4-bit pages 5 where there are no more: their weights' three pieces then lie side by side in the 16 columns of a
// product.  (Two pieces side by side for up to 8 columns gain nothing: 8 query heads a KV head, fp16, 64.6 us and 65.9 with 16 columns, bf16 62.6 and 62.4.)
template <int D, bool F16, bool FP4, int COLS = 16> struct Geo {
    static constexpr int kSlots = COLS == 5 ? 3 : 1;
    static constexpr int NB = D / kBlock, C = chunk_of(D), VL = D / C;        // VL lanes of 16 hold dims of V
    static constexpr int kTiles = 2, kStep = 16 * kTiles;           // rows of a step
    static constexpr int J = D / 32;                                          // products over the dims of a row
    // 4 bits: lane g holds dims D / 4 * g on, J words of a row; one scale byte or two if that is no more than a block or two
    static constexpr int kScales = D == 64 || D == 128 ? 1 : D == 256 ? 2 : J;
    static constexpr int kVWords = FP4 ? C / 2 : 2 * C;
    // fp16 weights are of up to 2^14, so that their second piece does not run out of exponents
    static constexpr bool kHalfP = F16 && !FP4;
    static constexpr float kShift = kHalfP ? 14.f : 0.f;
    static constexpr int kPieces = kHalfP ? 2 : 3, kSets = (kPieces + kSlots - 1) / kSlots;   // products a pair of a row's dims
};

// What a lane (n = lane % 16, g = lane / 16) holds of a step's rows.
template <int D, bool F16, bool FP4> struct Rows {
    using Q = Geo<D, F16, FP4>;
    uint32_t k[Q::kTiles][FP4 ? Q::J : 4 * Q::J];   // row n of a tile; 4 bits: dims D / 4 * g + 8 j .., 16 bits: 32 j + 8 g ..
    uint32_t ks[Q::kScales];             // 4 bits: scale bytes of rows n, 16 + n, 32 + n, 48 + n of the lane's blocks
    uint32_t v[Q::kTiles][Q::kVWords];   // rows 4 g .. 4 g + 3 of a tile, dims C n .. C n + C - 1
    uint32_t vs[Q::kTiles];              // 4 bits: scale bytes of those rows, a word a tile
};

// N words from an address that is a multiple of the largest load that divides them.  ONCE: no cache keeps them; not where a wavefront's load takes
// parts of lines whose rest the next one takes (head dims from 192 on: 36 x 8 x 4096 rows of 256 dims of 4 bits 78.8 us that way, 74.5 without; of 128 dims
// of 4 bits 61.4 and 69.3).
template <bool ONCE, typename T> __device__ __forceinline__ T load_from(const uint8_t *at)
{
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const T *>(at));
    else return *reinterpret_cast<const T *>(at);
}
template <int N, bool ONCE> __device__ __forceinline__ void load_words(uint32_t *w, const uint8_t *at)
{
    using u32x3 = unsigned int __attribute__((ext_vector_type(3), aligned(4)));
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const u32x4 x = load_from<ONCE, u32x4>(at + 4 * i);
            w[i] = x.x, w[i + 1] = x.y, w[i + 2] = x.z, w[i + 3] = x.w;
        }
    } else if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const u32x2 x = load_from<ONCE, u32x2>(at + 4 * i);
            w[i] = x.x, w[i + 1] = x.y;
        }
    } else {
        static_assert(N == 3, "1 1/2 blocks");
        const u32x3 x = *reinterpret_cast<const u32x3 *>(at);
        w[0] = x.x, w[1] = x.y, w[2] = x.z;
    }
}

template <int D, bool F16, bool FP4>
__device__ __forceinline__ void load_keys(Rows<D, F16, FP4> &f, const uint8_t *__restrict__ page, int half, int n, int g)
{
    using Q = Geo<D, F16, FP4>;
    if constexpr (FP4) {
        using P = Fp4Page<D>;
#pragma unroll
        for (int t = 0; t < Q::kTiles; ++t) load_words<Q::J, D <= 128>(f.k[t], page + P::k_code(half * Q::kStep + 16 * t + n, D / 4 * g));
#pragma unroll
        for (int i = 0; i < Q::kScales; ++i)
            f.ks[i] = *reinterpret_cast<const uint32_t *>(page + P::k_scale(n, (D / 4 * g + (Q::kScales == Q::J ? 8 : 32) * i) / kBlock));
    } else {
        using P = WidePage<D>;
#pragma unroll
        for (int t = 0; t < Q::kTiles; ++t)
#pragma unroll
            for (int b = 0; b < Q::J; ++b) load_words<4, D <= 128>(f.k[t] + 4 * b, page + P::k(half * Q::kStep + 16 * t + n, 32 * b + 8 * g));
    }
}
template <int D, bool F16, bool FP4>
__device__ __forceinline__ void load_values(Rows<D, F16, FP4> &f, const uint8_t *__restrict__ page, int half, int n, int g)
{
    using Q = Geo<D, F16, FP4>;
    const int vn = min(n, Q::VL - 1);                                     // lanes without dims of V take another's
    if constexpr (FP4) {
        using P = Fp4Page<D>;
#pragma unroll
        for (int t = 0; t < Q::kTiles; ++t) load_words<Q::kVWords, D <= 128>(f.v[t], page + P::v_code(half * Q::kStep + 16 * t + 4 * g, Q::C * vn));
        load_words<Q::kTiles, D <= 128>(f.vs, page + P::v_scale(half * Q::kStep + 4 * g, Q::C * vn / kBlock));
    } else {
        using P = WidePage<D>;
#pragma unroll
        for (int t = 0; t < Q::kTiles; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) load_words<Q::C / 2, D <= 128>(f.v[t] + i * (Q::C / 2), page + P::v(half * Q::kStep + 16 * t + 4 * g + i, Q::C * vn));
    }
}

// A column's query as the products take it: word j of a lane holds the dims that k's does.  A negative scale's sign goes to the query (flip:
// 0x80008000), so that the largest logit is that of the largest product.
// An fp16 query against 4-bit keys is two bf16 pieces.
template <int D, bool F16, bool FP4> struct Query {
    u32x4 w[F16 && FP4 ? 2 : 1][D / 32];
};

template <int D, bool F16, bool FP4>
__device__ __forceinline__ void load_query(Query<D, F16, FP4> &f, const uint16_t *__restrict__ row, bool there, uint32_t flip, int g)
{
    using Q = Geo<D, F16, FP4>;
#pragma unroll
    for (int j = 0; j < Q::J; ++j) {
        const int dim = FP4 ? D / 4 * g + 8 * j : 32 * j + 8 * g;
        u32x4 x = there ? *reinterpret_cast<const u32x4 *>(row + dim) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] ^= flip;
        if constexpr (F16 && FP4) {                                       // 11 bits: eight, and the three that are left
            float v[8], rest[8];
            unpack8<true>(x, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float cut = __uint_as_float(__float_as_uint(v[i]) & 0xffff0000u);
                rest[i] = v[i] - cut;
                v[i] = cut;
            }
            f.w[0][j] = pack8<false>(v);
            f.w[1][j] = pack8<false>(rest);
        } else {
            f.w[0][j] = x;
        }
    }
}

// The conversions read a scale's exponent field alone: the byte is moved there, whatever comes with it.
__device__ __forceinline__ float scale_bits(uint32_t word, int byte) { return __uint_as_float(byte < 3 ? word << (23 - 8 * byte) : word >> 1); }

// Two dims (2 i, 2 i + 1 of the word) as bf16
__device__ __forceinline__ uint32_t two_codes(uint32_t w, float scale, int i)
{
    switch (i) {
    case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    }
}

// c + the product of 16 x 32 and 32 x 16 values of fp16 (HALF) or bf16
template <bool HALF> __device__ __forceinline__ f32x4 product(const u32x4 &a, const u32x4 &b, f32x4 c)
{
    if constexpr (HALF) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// s[t][i]: <k, q> of row 16 t + 4 g + i and column n
template <int D, bool F16, bool FP4>
__device__ __forceinline__ void key_products(const Rows<D, F16, FP4> &f, const Query<D, F16, FP4> &q, int half, f32x4 (&s)[Geo<D, F16, FP4>::kTiles])
{
    using Q = Geo<D, F16, FP4>;
#pragma unroll
    for (int t = 0; t < Q::kTiles; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < Q::J; ++j)
#pragma unroll
        for (int t = 0; t < Q::kTiles; ++t) {
            if constexpr (FP4) {
                const float scale = scale_bits(f.ks[Q::kScales == Q::J ? j : j * Q::kScales / Q::J], Q::kTiles * half + t);
                u32x4 x;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = two_codes(f.k[t][j], scale, i);
                if constexpr (F16) s[t] = product<false>(x, q.w[1][j], s[t]);
                s[t] = product<false>(x, q.w[0][j], s[t]);
            } else {
                s[t] = product<F16>(u32x4{f.k[t][4 * j], f.k[t][4 * j + 1], f.k[t][4 * j + 2], f.k[t][4 * j + 3]}, q.w[0][j], s[t]);
            }
        }
}

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Running state of 16 columns: lane (n, g) holds column n's maximum, its own rows' share of the sum, and the weighted values of dims
// (4 g + i) C + t in o[t][i].
template <int D, bool F16, bool FP4, int COLS> struct State {
    using Q = Geo<D, F16, FP4, COLS>;
    float m, l;
    f32x4 o[Q::C], sums;                 // COLS = 5: the sum of a column's piece in every element of sums, l is not used
    __device__ __forceinline__ void clear()
    {
        m = kNone, l = 0.f, sums = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < Q::C; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
};

// The end of a unit's rows.  rel: rows from the half's first one on, lim: those that the lane's column sees, least: those that all columns see.
// Rows that a column does not see get the product -inf, so weight 0; V of rows that are not there becomes 0 or 1, since 0 times NaN is NaN.  So it does
// where a row that only later tokens see holds a NaN or infinity (in 4 bits: a block of a scale from 2^126 on, whose larger codes are beyond bf16), whose
// columns get a NaN for a product instead.
template <int D, bool F16, bool FP4>
__device__ __forceinline__ void mask_rows(Rows<D, F16, FP4> &f, f32x4 (&s)[Geo<D, F16, FP4>::kTiles], int g, int rel, int lim, int least)
{
    using Q = Geo<D, F16, FP4>;
#pragma unroll
    for (int t = 0; t < Q::kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 16 * t + 4 * g + i;
            bool clear = row >= rel, poison = false;
            if (least < rel) {                                             // several tokens
                bool odd = false;
                if constexpr (FP4) odd = (f.vs[t] >> (8 * i) & 255u) >= 253u;
                else
#pragma unroll
                    for (int k = 0; k < Q::C / 2; ++k) {
                        const uint32_t x = f.v[t][i * (Q::C / 2) + k], e = F16 ? 0x7c00u : 0x7f80u;
                        odd |= (x & e) == e || (x >> 16 & e) == e;
                    }
                const unsigned long long lanes = __ballot(odd);            // all dims of the row: the 16 lanes of this g
                poison = (lanes >> (16 * g) & 0xffffull) != 0ull && row >= least && row < rel;
                clear |= poison;
            }
            if constexpr (FP4) f.vs[t] = clear ? (f.vs[t] & ~(255u << (8 * i))) | 127u << (8 * i) : f.vs[t];
            else
#pragma unroll
                for (int k = 0; k < Q::C / 2; ++k) f.v[t][i * (Q::C / 2) + k] = clear ? 0u : f.v[t][i * (Q::C / 2) + k];
            s[t][i] = row >= lim ? -INFINITY : poison ? __uint_as_float(0x7fc00000u) : s[t][i];
        }
}

__device__ __forceinline__ bool sees_row(int row, int rel, int upto, int from, int front) { return row < rel && ((row < upto && row >= from) || row < front); }
// The same by rules: a column sees rows from .. upto - 1 of the half and those before `front`, all columns do all_from .. and so on.  Where a row that not all columns see
// holds a NaN or infinity, its V becomes 0 or 1, and the columns that do see it get a NaN for a product.
template <int D, bool F16, bool FP4>
__device__ __forceinline__ void mask_rows_by_rules(Rows<D, F16, FP4> &f, f32x4 (&s)[Geo<D, F16, FP4>::kTiles], int g, int rel, int upto, int from, int front, int all_upto, int all_from,
                                                   int all_front)
{
    using Q = Geo<D, F16, FP4>;
#pragma unroll
    for (int t = 0; t < Q::kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 16 * t + 4 * g + i;
            bool odd = false;
            if constexpr (FP4) odd = (f.vs[t] >> (8 * i) & 255u) >= 253u;
            else
#pragma unroll
                for (int k = 0; k < Q::C / 2; ++k) {
                    const uint32_t x = f.v[t][i * (Q::C / 2) + k], e = F16 ? 0x7c00u : 0x7f80u;
                    odd |= (x & e) == e || (x >> 16 & e) == e;
                }
            const unsigned long long lanes = __ballot(odd);                // all dims of the row: the 16 lanes of this g
            const bool by_all = row < rel && ((row < all_upto && row >= all_from) || row < all_front);
            const bool poison = (lanes >> (16 * g) & 0xffffull) != 0ull && !by_all, clear = row >= rel || poison;
            if constexpr (FP4) f.vs[t] = clear ? (f.vs[t] & ~(255u << (8 * i))) | 127u << (8 * i) : f.vs[t];
            else
#pragma unroll
                for (int k = 0; k < Q::C / 2; ++k) f.v[t][i * (Q::C / 2) + k] = clear ? 0u : f.v[t][i * (Q::C / 2) + k];
            s[t][i] = !sees_row(row, rel, upto, from, front) ? -INFINITY : poison ? __uint_as_float(0x7fc00000u) : s[t][i];
        }
}

// Products to logits in powers of two, by cap and distance.  from: rows between the lane's first one and its token's.
template <int D, bool F16, bool FP4>
__device__ __forceinline__ void bend_products(const AttendArgs &a, f32x4 (&s)[Geo<D, F16, FP4>::kTiles], float most, float from, float slope)
{
    constexpr int N = 4 * Geo<D, F16, FP4>::kTiles;
    float z[N];
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = s[i / 4][i % 4];
    if (a.cap.cap_log2 != 0.f) {
        bend(z, most, a.cap);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] *= a.scale_log2;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) s[i / 4][i % 4] = a.slopes ? fmaf(-slope, fabsf(from - (float)(16 * (i / 4) + i % 4)), z[i]) : z[i];
}

// WHOLE: weights in all the pieces that hold their 24 bits (fp16 rows of 16-bit pages: 22); otherwise rounded to the 16 bits that the output has (fp16 rows of 4-bit
// pages: to two pieces of bf16), a third of the products with V.
template <int D, bool F16, bool FP4, int COLS, bool WHOLE>
__device__ __forceinline__ void accumulate(State<D, F16, FP4, COLS> &st, const Rows<D, F16, FP4> &f, const f32x4 (&products)[Geo<D, F16, FP4>::kTiles],
                                           float scale_log2, int slot)
{
    using Q = Geo<D, F16, FP4, COLS>;
    float p[4 * Q::kTiles], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4 * Q::kTiles; ++i) {
        p[i] = products[i / 4][i % 4];
        top = fmaxf(top, p[i]);
    }
    top *= scale_log2;                                                     // (positive, see load_query)
    bool far = false, own = false;
    if (__any(top > st.m || fabsf(st.m) >= kFar)) {                        // seldom after a unit's first steps
        auto larger = [](float a, float b) { return fmaxf(a, b); };
        top = swap_reduce<32>(swap_reduce<16>(top, larger), larger);
        const float m = fmaxf(top, st.m), f0 = __builtin_amdgcn_exp2f(st.m - m);
        st.m = m;
        st.l *= f0;
#pragma unroll
        for (int i = 0; i < 4; ++i) st.sums[i] *= f0;
#pragma unroll
        for (int t = 0; t < Q::C; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) st.o[t][i] *= f0;
        own = fabsf(m) >= kFar && m > kNone;                               // (not where a column has seen no row yet)
        far = __any(own);
        if (far) {
#pragma clang fp contract(off)
#pragma unroll
            for (int i = 0; i < 4 * Q::kTiles; ++i) p[i] = WHOLE || own ? p[i] * scale_log2 - m : p[i];
        }
    }
    // By rules each column by itself: what others see leaves its weights as they are.
    const bool rounded = WHOLE ? far : own;
    const float base = Q::kShift - (rounded ? 0.f : st.m), factor = rounded ? 1.f : scale_log2;
#pragma unroll
    for (int i = 0; i < 4 * Q::kTiles; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(p[i], factor, base));
    // dims 2 k and 2 k + 1 of row 16 t + 4 g + i, next to each other
    auto values = [&](int t, int i, int k) {
        const int at = i * (Q::C / 2) + k;
        if constexpr (FP4) return two_codes(f.v[t][at / 4], scale_bits(f.vs[t], i), at % 4);
        else return f.v[t][at];
    };
    // The three pieces of a weight are its bits 24 .. 17, 16 .. 9 and 8 .. 1, the differences between it cut off behind them: exact, and cut to bf16 as
    // they are.  A lane of COLS = 5 takes the one of its slot.
    constexpr uint32_t kTop = 0xffff0000u, kMid = 0xffffff00u;
    auto between = [](float x, uint32_t upto, uint32_t above) {
        return __float_as_uint(__uint_as_float(__float_as_uint(x) & upto) - __uint_as_float(__float_as_uint(x) & above));
    };
    if constexpr (COLS == 5) {
        static_assert(WHOLE, "three pieces side by side");
        // A row's two dims stay side by side, as a product's two rows: beside (piece, 0) for the first dim, (0, piece) for the second.  Twice the
        // products, of which there are few, and no exchange of halves between rows' words.  The sum of the weights is one more product, with ones.
        constexpr uint32_t one = 0x3f803f80u;
        const uint32_t upto = slot == 0 ? kTop : slot == 1 ? kMid : ~0u, above = slot == 0 ? 0u : slot == 1 ? kTop : kMid;
#pragma unroll
        for (int t = 0; t < Q::kTiles; ++t) {
            u32x4 low, high;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t own = between(p[4 * t + i], upto, above);
                high[i] = own & kTop;                                      // (a piece under 2^-126 has bits down there)
                low[i] = own >> 16;
            }
            st.sums = product<false>(u32x4{one, one, one, one}, low, st.sums);
#pragma unroll
            for (int k = 0; k < Q::C / 2; ++k) {
                const u32x4 v = {values(t, 0, k), values(t, 1, k), values(t, 2, k), values(t, 3, k)};
                st.o[2 * k] = product<false>(v, low, st.o[2 * k]);
                st.o[2 * k + 1] = product<false>(v, high, st.o[2 * k + 1]);
            }
        }
    } else {
        float l = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * Q::kTiles; ++i) l += p[i];
        st.l += l;
        // the 32 rows of two tiles: words of two rows' weights, a piece at a time
        constexpr int kSets = WHOLE ? Q::kSets : F16 && FP4 ? 2 : 1;
        u32x4 w[kSets];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float a = p[2 * j], b = p[2 * j + 1];
            if constexpr (!WHOLE && kSets == 1) {
                if constexpr (F16) w[0][j] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
                else w[0][j] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
            } else if constexpr (!WHOLE) {
                w[0][j] = high_halves(__float_as_uint(a), __float_as_uint(b));
                w[1][j] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)__uint_as_float(between(a, ~0u, kTop)), (__bf16)__uint_as_float(between(b, ~0u, kTop))});
            } else if constexpr (Q::kHalfP) {
                const f16x2 hi = {(_Float16)a, (_Float16)b}, lo = {(_Float16)(a - (float)hi.x), (_Float16)(b - (float)hi.y)};
                w[0][j] = __builtin_bit_cast(uint32_t, hi), w[1][j] = __builtin_bit_cast(uint32_t, lo);
            } else {
                w[0][j] = high_halves(__float_as_uint(a), __float_as_uint(b));
                w[1][j] = high_halves(between(a, kMid, kTop), between(b, kMid, kTop));
                w[2][j] = high_halves(between(a, ~0u, kMid), between(b, ~0u, kMid));
            }
        }
#pragma unroll
        for (int k = 0; k < Q::C / 2; ++k) {
            uint32_t x[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) x[r] = values(r / 4, r % 4, k);
            const u32x4 lo = {low_halves(x[0], x[1]), low_halves(x[2], x[3]), low_halves(x[4], x[5]), low_halves(x[6], x[7])};
            const u32x4 hi = {high_halves(x[0], x[1]), high_halves(x[2], x[3]), high_halves(x[4], x[5]), high_halves(x[6], x[7])};
#pragma unroll
            for (int c = kSets - 1; c >= 0; --c) {
                st.o[2 * k] = product<Q::kHalfP>(lo, w[c], st.o[2 * k]);
                st.o[2 * k + 1] = product<Q::kHalfP>(hi, w[c], st.o[2 * k + 1]);
            }
        }
    }
}

// Which parts the workspace holds of a unit: one for every stretch x .. y - 1 that it lies in, but one (numbered as its first) for every
// workgroup's kWaves stretches from group a to b - 1, which lie in the unit altogether.
struct Parts {
    int x, y, a, b;
    __device__ int count() const { return a < b ? (kWaves * a - x) + (b - a) + (y - kWaves * b > 0 ? y - kWaves * b : 0) : y - x; }
    __device__ int number(int i) const                                    // the stretch of the i-th part
    {
        if (a >= b) return x + i;
        const int front = kWaves * a - x;
        return i < front ? x + i : i < front + (b - a) ? kWaves * (a + i - front) : kWaves * b + (i - front - (b - a));
    }
};
// All units' pages in n stretches, the first `rem` one page longer than the others.  (All of the rounded-up length left up to one wavefront in sixteen
// without pages where the stretches are short: twelve or thirteen pages each.)
struct Cut {
    uint32_t base, rem;
    __device__ Cut() {}
    __device__ Cut(uint32_t total, uint32_t n) : base(total / n), rem(total - total / n * n) {}
    __device__ uint32_t first(uint32_t i) const { return i * base + min(i, rem); }
    __device__ uint32_t of(uint32_t at) const                              // the stretch that holds a page
    {
        const uint32_t wide = rem * (base + 1);
        return at < wide ? at / (base + 1) : rem + (at - wide) / base;
    }
};
// of a unit whose c > 0 pages are the at-th on; total: of all units
__device__ __forceinline__ Parts parts_of(uint32_t at, uint32_t c, const Cut &cut, uint32_t total)
{
    Parts p;
    p.x = (int)cut.of(at);
    p.y = (int)cut.of(at + c - 1) + 1;
    const int whole = p.x + (cut.first(p.x) < at ? 1 : 0), upto = p.y - (cut.first(p.y) > at + c ? 1 : 0);   // the stretches that lie in the unit altogether
    p.a = (whole + kWaves - 1) / kWaves;
    p.b = at + c == total ? (p.y + kWaves - 1) / kWaves : upto / kWaves;   // (behind the last page stretches are empty)
    return p;
}

// Where a wavefront's stretch begins.  The pages of all units are counted in their order.
struct Place {
    uint32_t total;
    Cut cut;
    int unit, unit0;                     // the unit that holds the stretch's first page, and that of the workgroup's first stretch
    uint32_t first;                      // the first page of `unit`
    bool joined;                         // all of the workgroup's pages lie in unit0: its wavefronts' parts become one
};
constexpr int kUnitsLane = 8;

__device__ __forceinline__ int prefix_of(const AttendArgs &a, int u, int len) { return a.prefix ? max(0, min(a.prefix[u / a.H], len)) : 0; }
// the pages that a unit's tokens see
template <bool RULES> __device__ __forceinline__ uint32_t pages_of(const AttendArgs &a, int u)
{
    const int len = clamp_len(a.lens[u], a.max_pages);
    if constexpr (RULES) return (uint32_t)seen_pages(len - a.n_new, len - 1, a.window, prefix_of(a, u, len)).count;
    else return (uint32_t)(len + kRows - 1) / kRows;
}
__device__ __forceinline__ bool plans() { return blockIdx.x == 0 && blockIdx.y == 0; }

// Up to 512 units: every wavefront counts them by itself, all lengths asked for at once and no barrier.
template <bool RULES> __device__ __forceinline__ Place placed_by_wave(const AttendArgs &a, int w)
{
    const int lane = threadIdx.x & (kWave - 1);
    uint32_t c[kUnitsLane], at[kUnitsLane];
#pragma unroll
    for (int k = 0; k < kUnitsLane; ++k) c[k] = k * kWave + lane < a.n_units ? pages_of<RULES>(a, k * kWave + lane) : 0u;
    Place p;
    p.total = 0u;
#pragma unroll
    for (int k = 0; k < kUnitsLane; ++k) {
        if (k * kWave >= a.n_units) break;
        const uint32_t incl = wave_prefix_sum(c[k]);
        at[k] = p.total + incl - c[k];
        p.total += (uint32_t)__builtin_amdgcn_readlane((int)incl, kWave - 1);
    }
    const uint32_t stretches = gridDim.x * kWaves;
    p.cut = Cut(p.total, stretches);
    const uint32_t lo0 = p.cut.first(blockIdx.x * kWaves), lo = p.cut.first(blockIdx.x * kWaves + w), hi = p.cut.first((blockIdx.x + 1) * kWaves);
    p.unit = p.unit0 = 0, p.first = 0u, p.joined = false;
#pragma unroll
    for (int k = 0; k < kUnitsLane; ++k) {
        if (k * kWave >= a.n_units) break;
        const unsigned long long mine = __ballot(at[k] <= lo && lo < at[k] + c[k]), groups = __ballot(at[k] <= lo0 && lo0 < at[k] + c[k]);
        if (mine) {
            const int l = __builtin_ctzll(mine);
            p.unit = k * kWave + l;
            p.first = (uint32_t)__builtin_amdgcn_readlane((int)at[k], l);
        }
        if (groups) {
            const int l = __builtin_ctzll(groups);
            p.unit0 = k * kWave + l;
            p.joined = (uint32_t)__builtin_amdgcn_readlane((int)(at[k] + c[k]), l) >= hi;
        }
        if (plans() && w == 0 && k * kWave + lane < a.n_units) a.plan[k * kWave + lane] = c[k] ? parts_of(at[k], c[k], p.cut, p.total) : Parts{0, 0, 0, 0};
    }
    return p;
}

// More units: the workgroup's threads count a share of them each.
template <bool RULES> __device__ __forceinline__ Place placed_by_workgroup(const AttendArgs &a, int w)
{
    __shared__ uint32_t wsum[kWaves], first[kWaves];
    __shared__ int unit[kWaves], joined;
    const int tid = threadIdx.x, per = (a.n_units + kThreads - 1) / kThreads, u0 = min(tid * per, a.n_units), u1 = min(u0 + per, a.n_units);
    uint32_t mine = 0u;
    for (int u = u0; u < u1; ++u) mine += pages_of<RULES>(a, u);
    uint32_t at = wave_prefix_sum(mine) - mine;
    if ((tid & (kWave - 1)) == kWave - 1) wsum[w] = at + mine;
    if (tid < kWaves) unit[tid] = 0, first[tid] = 0u;
    __syncthreads();
    Place p;
    p.total = 0u;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        at += i < w ? wsum[i] : 0u;
        p.total += wsum[i];
    }
    const uint32_t stretches = gridDim.x * kWaves;
    p.cut = Cut(p.total, stretches);
    const uint32_t lo0 = p.cut.first(blockIdx.x * kWaves), hi = p.cut.first((blockIdx.x + 1) * kWaves);
    if (plans() || (at < hi && at + mine > lo0)) {
        for (int u = u0; u < u1; ++u) {
            const uint32_t c = pages_of<RULES>(a, u);
            if (plans()) a.plan[u] = c ? parts_of(at, c, p.cut, p.total) : Parts{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < kWaves; ++i)
                if (const uint32_t lo = p.cut.first(blockIdx.x * kWaves + i); at <= lo && lo < at + c) {
                    unit[i] = u;
                    first[i] = at;
                    if (i == 0) joined = at + c >= hi;
                }
            at += c;
        }
    }
    __syncthreads();
    p.unit = __builtin_amdgcn_readfirstlane(unit[w]), p.unit0 = __builtin_amdgcn_readfirstlane(unit[0]);
    p.first = (uint32_t)__builtin_amdgcn_readfirstlane((int)first[w]);
    p.joined = __builtin_amdgcn_readfirstlane(joined) != 0;
    return p;
}

// Older wavefronts of a SIMD are served first, and stretches are equally long: a compute unit's first workgroup was done after 40 us, its third after 51
// (36 x 8 x 8192 rows of 4 bits).  So those with more of their stretch left go first, by quarters: 60.4 -> 60.1 us, with 8 query heads a KV head 66.1 ->
// 62.5, of 64 dims 38.3 -> 35.9, of 256 dims of 16 bits 137 -> 131.
__device__ __forceinline__ void by_what_is_left(uint32_t left, uint32_t run)
{
    if (4u * left > 3u * run) __builtin_amdgcn_s_setprio(3);
    else if (2u * left > run) __builtin_amdgcn_s_setprio(2);
    else if (4u * left > run) __builtin_amdgcn_s_setprio(1);
    else __builtin_amdgcn_s_setprio(0);
}

// Wavefronts of a workgroup that has a unit to itself.
constexpr int kUnitWaves = 8;

// grid: (stretches / kWaves, groups of columns).  ALONE: (units, groups of columns), a workgroup a unit, whose pages its wavefronts share out; nothing is left to join.
template <int D, bool F16, bool FP4, int COLS, bool RULES, bool ALONE = false>
__global__ __launch_bounds__((ALONE ? kUnitWaves * kWave : kThreads), (ALONE ? 2 : groups_at_once(D))) void pages_attend_kernel(const AttendArgs a)
{
    using Q = Geo<D, F16, FP4, COLS>;
    constexpr int kWaves = ALONE ? kUnitWaves : nkv::kWaves, kThreads = kWaves * kWave;
    constexpr int kBytes = FP4 ? Fp4Page<D>::kBytes : WidePage<D>::kBytes;
    __shared__ __align__(16) float lds_o[kWaves][16][D + 4];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    __builtin_amdgcn_s_setprio(3);
    Place at;
    if constexpr (ALONE) {
        at.unit = at.unit0 = blockIdx.x, at.joined = true, at.first = 0u;
    } else {
        at = a.n_units <= kWave * kUnitsLane ? placed_by_wave<RULES>(a, w) : placed_by_workgroup<RULES>(a, w);
        const uint32_t group_lo = at.cut.first(blockIdx.x * kWaves);
        if (group_lo >= at.total) return;
    }
    // ---- columns ----
    const int cols = a.n_new * a.G, col0 = blockIdx.y * COLS, col = col0 + n % COLS, slot = n / COLS;
    const bool there = col < cols;
    const int token = (there ? col : cols - 1) / a.G, head = (there ? col : cols - 1) - token * a.G;

    const uint32_t stretch = blockIdx.x * kWaves + w, all = ALONE ? pages_of<RULES>(a, at.unit) : 0u;
    const uint32_t lo = ALONE ? all * w / kWaves : at.cut.first(stretch), hi = ALONE ? all * (w + 1) / kWaves : at.cut.first(stretch + 1);
    int u = at.unit;
    uint32_t step = lo - at.first;                                         // page of the unit
    const bool joined = at.joined;
    const int here = min(COLS, cols - col0);
    // columns [0, here) of what `waves` wavefronts left, from `first` on, by `threads` threads, to the workspace
    auto write = [&](int first, int waves, int number, int unit, int thread, int threads) {
        float *dst = a.part + (((int64_t)number + unit) * cols + col0) * (D + 4);
        for (int idx = thread; idx < here * (D / 4); idx += threads) {
            const int c = idx / (D / 4), e = (idx - c * (D / 4)) * 4;
            float mm = kNone, ll = 0.f;
            f32x4 oo = {0.f, 0.f, 0.f, 0.f};
            for (int i = first; i < first + waves; ++i) mm = fmaxf(mm, lds_o[i][c][D]);
            for (int i = first; i < first + waves; ++i) {
                const float f = __builtin_amdgcn_exp2f(lds_o[i][c][D] - mm);
                f32x4 x = *reinterpret_cast<const f32x4 *>(&lds_o[i][c][e]);
#pragma unroll
                for (int k = 1; k < Q::kSlots; ++k) {
                    const f32x4 y = *reinterpret_cast<const f32x4 *>(&lds_o[i][c + k * COLS][e]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] += y[r];
                }
                float l = lds_o[i][c][D + 1];
                if constexpr (COLS == 5)
#pragma unroll
                    for (int k = 1; k < Q::kSlots; ++k) l += lds_o[i][c + k * COLS][D + 1];
                ll = fmaf(f, l, ll);
#pragma unroll
                for (int k = 0; k < 4; ++k) oo[k] = fmaf(f, x[k], oo[k]);
            }
            if constexpr (ALONE) {                                         // (as pages_combine_kernel does)
                const int t = (col0 + c) / a.G, sq = unit / a.H;
                const int64_t row = ((int64_t)sq * a.n_new + t) * a.H * a.G + (unit - sq * a.H) * a.G + (col0 + c - t * a.G);
                const bool none = ll == 0.f;                               // (NaN is handed on)
#pragma unroll
                for (int k = 0; k < 4; ++k) oo[k] = none ? 0.f : oo[k] / ll;
                using Out = std::conditional_t<F16, _Float16, __bf16>;
                using Out4 = Out __attribute__((ext_vector_type(4)));
                *reinterpret_cast<Out4 *>((Out *)a.out + row * D + e) = Out4{(Out)oo[0], (Out)oo[1], (Out)oo[2], (Out)oo[3]};
                if (a.lse && e == 0) a.lse[row] = none ? -INFINITY : (mm + log2f(ll)) * kLn2;
                continue;
            }
            *reinterpret_cast<f32x4 *>(dst + c * (D + 4) + e) = oo;
            if (e == 0) {
                dst[c * (D + 4) + D] = mm;
                dst[c * (D + 4) + D + 1] = ll;
            }
        }
    };
    // ---- the stretch, unit by unit ----
    uint32_t i = lo;
    do {
        Query<D, F16, FP4> q;
        State<D, F16, FP4, COLS> st;
        st.clear();
        const int len = clamp_len(a.lens[u], a.max_pages), sq = u / a.H, h = u - sq * a.H;
        const int32_t *table = a.table + (int64_t)u * a.max_pages;
        Seen seen{};
        int prefix = 0;
        float slope = 0.f;
        if constexpr (RULES) {
            if (a.slopes) slope = a.slopes[h * a.G + head] * kToLog2;
            prefix = prefix_of(a, u, len);
            seen = seen_pages(len - a.n_new, len - 1, a.window, prefix);
        }
        const uint32_t left = (RULES ? (uint32_t)seen.count : (uint32_t)(len + kRows - 1) / kRows) - step, end = i < hi ? step + min(hi - i, left) : step;
        if (i < hi) load_query<D, F16, FP4>(q, a.q + (((int64_t)sq * a.n_new + token) * a.H * a.G + h * a.G + head) * D, there && !a.flat, a.flip, g);
        i += end - step;
        auto page_at = [&](uint32_t at) { return RULES ? (uint32_t)seen.page((int)at) : at; };
        auto id_of = [&](uint32_t at) { return at < end ? table[page_at(at)] : -1; };
        auto page_of = [&](int id) { return a.pool + (int64_t)(id >= 0 && id < a.n_pages ? id : 0) * kBytes; };
        int id = id_of(step), next = id_of(step + 1);
        const uint8_t *page = page_of(id);
        // A half's rows, while the next half's are on their way.  4 bits: in a second set of registers.  16 bits: in the same ones, keys as soon as their
        // products are made, values after theirs.  (Behind the last page: some page's.)
        Rows<D, F16, FP4> even, odd;
        auto take = [&](Rows<D, F16, FP4> &f, const int half, bool counts, auto keys_on, auto values_on) {
            const int row0 = (int)(page_at(step) * kRows) + half * Q::kStep, rel = len - row0, least = rel - (a.n_new - 1);
            const bool works = counts && rel > 0;                          // (a half without rows is loaded too: its bytes are the page's)
            f32x4 s[Q::kTiles];
            if (works) key_products<D, F16, FP4>(f, q, half, s);
            keys_on();
            if constexpr (RULES) {
                if (works) {
                    // all of the half's rows are seen by all tokens
                    const int r0 = len - a.n_new, r1 = len - 1;
                    const bool part = !(r0 >= 0 && rel >= Q::kStep && (row0 + Q::kStep <= prefix || (least >= Q::kStep && (a.window <= 0 || row0 > r1 - a.window))));
                    const int at = r0 + token, since = a.window > 0 ? max(at, 0) - a.window + 1 : 0;
                    const bool some = at >= 0, all = r0 >= 0;              // (a token in front of the unit's first row sees nothing)
                    const int upto = some ? at + 1 - row0 : 0, from = some ? since - row0 : 0, front = some ? prefix - row0 : 0;
                    if (a.bent) {
                        float most = 0.f;
                        if (a.cap.cap_log2 != 0.f)
#pragma unroll
                            for (int k = 0; k < 4 * Q::kTiles; ++k) most = !part || sees_row(16 * (k / 4) + 4 * g + k % 4, rel, upto, from, front) ? fmaxf(most, fabsf(s[k / 4][k % 4])) : most;
                        bend_products<D, F16, FP4>(a, s, most, (float)(len - a.n_new + token - row0 - 4 * g), slope);
                    }
                    if (part)
                        mask_rows_by_rules<D, F16, FP4>(f, s, g, rel, upto, from, front, all ? least : 0, all && a.window > 0 ? r1 - a.window + 1 - row0 : 0, all ? prefix - row0 : 0);
                    accumulate<D, F16, FP4, COLS, false>(st, f, s, a.bent ? 1.f : a.scale_log2, slot);
                }
            } else if (works) {
                if (least < Q::kStep) mask_rows<D, F16, FP4>(f, s, g, rel, least + token, least);
                accumulate<D, F16, FP4, COLS, true>(st, f, s, a.scale_log2, slot);
            }
            values_on();
        };
        if (step < end) {
            load_keys<D, F16, FP4>(even, page, 0, n, g);
            load_values<D, F16, FP4>(even, page, 0, n, g);
        }
        while (step < end) {
            const int after = id_of(step + 2);
            const bool counts = id >= 0 && id < a.n_pages;
            const uint8_t *const this_page = page;
            id = next, next = after, page = page_of(id);
            auto nothing = [] {};
            if constexpr (FP4) {
                load_keys<D, F16, FP4>(odd, this_page, 1, n, g);
                load_values<D, F16, FP4>(odd, this_page, 1, n, g);
                take(even, 0, counts, nothing, nothing);
                load_keys<D, F16, FP4>(even, page, 0, n, g);
                load_values<D, F16, FP4>(even, page, 0, n, g);
                take(odd, 1, counts, nothing, nothing);
            } else {
                take(even, 0, counts, [&] { load_keys<D, F16, FP4>(even, this_page, 1, n, g); }, [&] { load_values<D, F16, FP4>(even, this_page, 1, n, g); });
                take(even, 1, counts, [&] { load_keys<D, F16, FP4>(even, page, 0, n, g); }, [&] { load_values<D, F16, FP4>(even, page, 0, n, g); });
            }
            ++step;
            by_what_is_left(hi - i + end - step, hi - lo);
        }
        auto sum = [](float x, float y) { return x + y; };
        const float l = COLS == 5 ? st.sums[0] : swap_reduce<32>(swap_reduce<16>(st.l, sum), sum);
        float *mine_o = lds_o[w][n];
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (4 * g + r < Q::VL)
#pragma unroll
                for (int t = 0; t < Q::C; t += 4)
                    *reinterpret_cast<f32x4 *>(mine_o + (4 * g + r) * Q::C + t) = f32x4{st.o[t][r], st.o[t + 1][r], st.o[t + 2][r], st.o[t + 3][r]};
        if (g == 0) {
            mine_o[D] = st.m - Q::kShift;
            mine_o[D + 1] = l;
        }
        if (joined) break;
        __builtin_amdgcn_wave_barrier();                                   // (a wavefront's LDS accesses are done in their order)
        if (i > lo) write(w, 1, (int)stretch, u, lane, 64);
        __builtin_amdgcn_wave_barrier();
        step = 0;
        do ++u;
        while (i < hi && u < a.n_units - 1 && (RULES ? pages_of<RULES>(a, u) == 0u : a.lens[u] <= 0));
    } while (i < hi);
    if (!joined) return;
    __syncthreads();
    write(0, kWaves, blockIdx.x * kWaves, at.unit0, tid, kThreads);
}

// grid: a workgroup for every unit and column.  D / 4 threads for a part, kThreads / (D / 4) parts at a time, each slice of parts with a running
// maximum of its own; the slices are added up in their order.
// Out: float, __bf16 or _Float16.
template <int D, typename Out> __global__ __launch_bounds__(kThreads) void pages_combine_kernel(const float *__restrict__ part, const Parts *__restrict__ plan, int cols, int H,
                                                                                               int G, int n_new, Out *__restrict__ out, float *__restrict__ lse)
{
    constexpr int TH = D / 4, NS = kThreads / TH, U = 4;
    __shared__ float lds_m[NS], lds_l[NS];
    __shared__ __align__(16) float lds_o[NS][D];
    const int u = blockIdx.x / cols, col = blockIdx.x - u * cols, tid = threadIdx.x, e = tid % TH * 4, sl = tid / TH;
    const Parts of = plan[u];
    const int count = of.count();
    float m = kNone, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (sl < NS) {
        for (int i = sl; i < count; i += U * NS) {                         // U parts' loads at once
            f32x4 x[U];
            float pm[U], pl[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const float *p = part + (((int64_t)of.number(min(i + k * NS, count - 1)) + u) * cols + col) * (D + 4);
                x[k] = *reinterpret_cast<const f32x4 *>(p + e);
                pm[k] = p[D], pl[k] = p[D + 1];
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (i + k * NS >= count) break;
                const float mm = fmaxf(m, pm[k]), f = __builtin_amdgcn_exp2f(m - mm), h = __builtin_amdgcn_exp2f(pm[k] - mm);
                m = mm;
                l = fmaf(l, f, h * pl[k]);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = fmaf(o[r], f, h * x[k][r]);
            }
        }
        *reinterpret_cast<f32x4 *>(&lds_o[sl][e]) = o;
        if (e == 0) lds_m[sl] = m, lds_l[sl] = l;
    }
    __syncthreads();
    if (sl > 0) return;
#pragma unroll
    for (int i = 1; i < NS; ++i) m = fmaxf(m, lds_m[i]);
    l = 0.f, o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const float f = __builtin_amdgcn_exp2f(lds_m[i] - m);
        const f32x4 x = *reinterpret_cast<const f32x4 *>(&lds_o[i][e]);
        l = fmaf(f, lds_l[i], l);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = fmaf(f, x[k], o[k]);
    }
    const int s = u / H, h = u - s * H, t = col / G, g = col - t * G;
    const int64_t row = ((int64_t)s * n_new + t) * H * G + h * G + g;
    const bool none = l == 0.f;                                           // (NaN is handed on)
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = none ? 0.f : o[k] / l;
    using Out4 = Out __attribute__((ext_vector_type(4)));
    *reinterpret_cast<Out4 *>(out + row * D + e) = Out4{(Out)o[0], (Out)o[1], (Out)o[2], (Out)o[3]};
    if (lse && e == 0) lse[row] = none ? -INFINITY : (m + log2f(l)) * kLn2;
}

unsigned groups_of(const nkv_pages &p)
{
    const int64_t most = (int64_t)p.n_seqs * p.H * p.max_pages;
    return (unsigned)std::min<int64_t>(256 * groups_at_once(p.d), (most + kWaves - 1) / kWaves);
}
size_t plan_bytes(const nkv_pages &p) { return ((size_t)p.n_seqs * p.H * sizeof(Parts) + 255) / 256 * 256; }

size_t columns_ws_bytes(const nkv_pages &p, int n_q_heads, int n_new)
{
    const size_t cols = (size_t)(n_q_heads / p.H) * n_new;
    return plan_bytes(p) + ((size_t)groups_of(p) * kWaves + (size_t)p.n_seqs * p.H) * cols * (p.d + 4) * sizeof(float);
}

// f(head dim, whether rows are fp16, whether pages are of 4 bits), as types
template <typename F> void for_rows(const nkv_pages &p, F f)
{
    for_head_dim(p.d, [&](auto dim) {
        const bool half = p.dtype == NKV_DTYPE_F16, four = p.format == NKV_PAGES_FP4;
        if (half && four) f(dim, std::true_type{}, std::true_type{});
        else if (half) f(dim, std::true_type{}, std::false_type{});
        else if (four) f(dim, std::false_type{}, std::true_type{});
        else f(dim, std::false_type{}, std::false_type{});
    });
}

// One launch, a workgroup a unit.
hipError_t launch_units(const AttendArgs &a, const nkv_pages &p, hipStream_t st)
{
    const dim3 grid(a.n_units, (unsigned)((a.G * a.n_new + 15) / 16));
    for_rows(p, [&](auto dim, auto f16, auto fp4) { pages_attend_kernel<decltype(dim)::value, decltype(f16)::value, decltype(fp4)::value, 16, true, true><<<grid, kUnitWaves * kWave, 0, st>>>(a); });
    return hipGetLastError();
}

// Both launches of a call; Out: what the output is of.
template <bool RULES, typename Out> hipError_t launch_columns(AttendArgs a, const nkv_pages &p, Out *out, float *lse, void *ws, hipStream_t st)
{
    a.plan = (Parts *)ws;
    a.part = (float *)((char *)ws + plan_bytes(p));
    const int cols = a.G * a.n_new;
    for_head_dim(p.d, [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        auto go = [&](auto f16, auto fp4) {
            constexpr bool F16 = decltype(f16)::value, FP4 = decltype(fp4)::value;
            if constexpr (std::is_same_v<Out, float> || std::is_same_v<Out, _Float16> == F16) {
                auto launch = [&](auto columns) {
                    constexpr int COLS = decltype(columns)::value;
                    pages_attend_kernel<D, F16, FP4, COLS, RULES><<<dim3(groups_of(p), (unsigned)((cols + COLS - 1) / COLS)), kThreads, 0, st>>>(a);
                };
                if constexpr (FP4 && !RULES) {                             // (16-bit rows are bound by memory with 16 columns too)
                    if (cols <= 5) return launch(std::integral_constant<int, 5>{});
                }
                launch(std::integral_constant<int, 16>{});
            }
        };
        using Yes = std::true_type;
        using No = std::false_type;
        const bool half = p.dtype == NKV_DTYPE_F16, four = p.format == NKV_PAGES_FP4;
        if (half && four) go(Yes{}, Yes{});
        else if (half) go(Yes{}, No{});
        else if (four) go(No{}, Yes{});
        else go(No{}, No{});
        pages_combine_kernel<D, Out><<<(unsigned)(a.n_units * cols), kThreads, 0, st>>>(a.part, a.plan, cols, a.H, a.G, a.n_new, out, lse);
    });
    return hipGetLastError();
}

}  // namespace
}  // namespace nkv
