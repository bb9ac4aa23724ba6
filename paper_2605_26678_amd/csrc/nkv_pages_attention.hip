// Attention of a sequence's last tokens over its pages (nkv_pages_attention).
//
// For unit u and its columns (token, query head): s_i = scale <q, k_i>, out = sum_i softmax(s)_i v_i over the rows that the column sees.
// Every row is read once for up to 16 columns and used for 4 d multiply-adds a column: bound by memory, if the rest keeps up.
// Both products go through the matrix cores, exactly:
//   S = K Q^T     4-bit values become bf16, which holds them exactly (an fp16 query then in two bf16 pieces); 16 x 16 x 32 products
//                 over a lane's dims in turn.  (The scaled product of 4-bit rows as they lie in the page and 8-bit pieces of a query
//                 loses bits of small terms beside large ones: up to 6e-6 of the terms' sum, 2e-7 in the mean.)
//   O^T = V^T P   two rows' dims are put side by side as the operand wants them; a weight is split into three bf16 pieces (two of fp16), which hold its 24 (22) bits.
// A column's running maximum, sum and weighted values stay in registers; with rows as the operands' other axis no lane
// exchange is needed between the products: the rows that a lane holds of S are those it holds of P, and V's rows are taken in that order.
//
// Work is cut into stretches of steps (64 rows of 4 bits, 32 of 16 bits) across units, one for every wavefront; a stretch's part of a unit
// goes to the workspace as (maximum, sum, weighted values) and pages_combine_kernel joins a unit's.
#include "nkv_pages.h"

#include <algorithm>

namespace nkv {
namespace {

using f32x4 = float __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256, kWaves = kThreads / 64, kCols = 16;
constexpr int kMostGroups = 512;         // workgroups: two for every compute unit
constexpr float kNone = -1.0e30f;        // running maximum before any row was seen
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ int clamp_len(int len, int max_pages) { return max(0, min(len, max_pages * kRows)); }

struct AttendArgs {
    const uint16_t *q;
    const uint8_t *pool;
    const int32_t *table, *lens;
    int32_t n_units, H, G, n_new, n_pages, max_pages;
    float scale_log2;
    int2 *plan;                          // per unit: its first part and the one behind its last
    float *part;                         // [part][column][D + 4]: weighted values, maximum, sum
};

template <int D, bool F16, bool FP4> struct Geo {
    static constexpr int NB = D / kBlock, C = chunk_of(D), VL = D / C;        // VL lanes of 16 hold dims of V
    static constexpr int kTiles = FP4 ? 4 : 2, kStep = 16 * kTiles;           // rows of a step
    static constexpr int J = D / 32;                                          // products over the dims of a row
    // 4 bits: lane g holds dims D / 4 * g on, J words of a row; one scale byte or two if that is no more than a block or two
    static constexpr int kScales = D == 64 || D == 128 ? 1 : D == 256 ? 2 : J;
    static constexpr int kVWords = FP4 ? C / 2 : 2 * C;
    // fp16 weights are of up to 2^14, so that their second piece does not run out of exponents
    static constexpr bool kHalfP = F16 && !FP4;
    static constexpr float kShift = kHalfP ? 14.f : 0.f;
    static constexpr int kPieces = kHalfP ? 2 : 3;
};

// What a lane (n = lane % 16, g = lane / 16) holds of a step's rows.
template <int D, bool F16, bool FP4> struct Rows {
    using Q = Geo<D, F16, FP4>;
    uint32_t k[Q::kTiles][FP4 ? Q::J : 4 * Q::J];   // row n of a tile; 4 bits: dims D / 4 * g + 8 j .., 16 bits: 32 j + 8 g ..
    uint32_t ks[Q::kScales];             // 4 bits: scale bytes of rows n, 16 + n, 32 + n, 48 + n of the lane's blocks
    uint32_t v[Q::kTiles][Q::kVWords];   // rows 4 g .. 4 g + 3 of a tile, dims C n .. C n + C - 1
    u32x4 vs;                            // 4 bits: scale bytes of those rows, a word a tile
};

// N words from an address that is a multiple of the largest load that divides them.
template <int N> __device__ __forceinline__ void load_words(uint32_t *w, const uint8_t *at)
{
    using u32x3 = unsigned int __attribute__((ext_vector_type(3), aligned(4)));
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(at + 4 * i));
            w[i] = x.x, w[i + 1] = x.y, w[i + 2] = x.z, w[i + 3] = x.w;
        }
    } else if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(at + 4 * i));
            w[i] = x.x, w[i + 1] = x.y;
        }
    } else {
        static_assert(N == 3, "1 1/2 blocks");
        const u32x3 x = *reinterpret_cast<const u32x3 *>(at);
        w[0] = x.x, w[1] = x.y, w[2] = x.z;
    }
}

template <int D, bool F16, bool FP4>
__device__ __forceinline__ void load_rows(Rows<D, F16, FP4> &f, const uint8_t *__restrict__ page, int half, int n, int g)
{
    using Q = Geo<D, F16, FP4>;
    const int vn = min(n, Q::VL - 1);                                     // lanes without dims of V take another's
    if constexpr (FP4) {
        using P = Fp4Page<D>;
#pragma unroll
        for (int t = 0; t < 4; ++t) load_words<Q::J>(f.k[t], page + P::k_code(16 * t + n, D / 4 * g));
#pragma unroll
        for (int i = 0; i < Q::kScales; ++i)
            f.ks[i] = *reinterpret_cast<const uint32_t *>(page + P::k_scale(n, (D / 4 * g + (Q::kScales == Q::J ? 8 : 32) * i) / kBlock));
#pragma unroll
        for (int t = 0; t < 4; ++t) load_words<Q::kVWords>(f.v[t], page + P::v_code(16 * t + 4 * g, Q::C * vn));
        f.vs = *reinterpret_cast<const u32x4 *>(page + P::v_scale(4 * g, Q::C * vn / kBlock));
    } else {
        using P = WidePage<D>;
#pragma unroll
        for (int t = 0; t < Q::kTiles; ++t)
#pragma unroll
            for (int b = 0; b < Q::J; ++b) load_words<4>(f.k[t] + 4 * b, page + P::k(half * Q::kStep + 16 * t + n, 32 * b + 8 * g));
#pragma unroll
        for (int t = 0; t < Q::kTiles; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) load_words<Q::C / 2>(f.v[t] + i * (Q::C / 2), page + P::v(half * Q::kStep + 16 * t + 4 * g + i, Q::C * vn));
    }
}

// A column's query as the products take it: word j of a lane holds the dims that k's does.
template <int D, bool F16, bool FP4> struct Query {
    u32x4 w[F16 && FP4 ? 2 : 1][D / 32];
};

template <int D, bool F16, bool FP4>
__device__ __forceinline__ void load_query(Query<D, F16, FP4> &f, const uint16_t *__restrict__ row, bool there, int g)
{
    using Q = Geo<D, F16, FP4>;
#pragma unroll
    for (int j = 0; j < Q::J; ++j) {
        const int dim = FP4 ? D / 4 * g + 8 * j : 32 * j + 8 * g;
        const u32x4 x = there ? *reinterpret_cast<const u32x4 *>(row + dim) : u32x4{0u, 0u, 0u, 0u};
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
__device__ __forceinline__ void key_products(const Rows<D, F16, FP4> &f, const Query<D, F16, FP4> &q, f32x4 (&s)[Geo<D, F16, FP4>::kTiles])
{
    using Q = Geo<D, F16, FP4>;
#pragma unroll
    for (int t = 0; t < Q::kTiles; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < Q::J; ++j)
#pragma unroll
        for (int t = 0; t < Q::kTiles; ++t) {
            if constexpr (FP4) {
                const float scale = scale_value(f.ks[Q::kScales == Q::J ? j : j * Q::kScales / Q::J] >> (8 * t) & 255u);
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
template <int D, bool F16, bool FP4> struct State {
    using Q = Geo<D, F16, FP4>;
    float m, l;
    f32x4 o[Q::C];
    __device__ __forceinline__ void clear()
    {
        m = kNone, l = 0.f;
#pragma unroll
        for (int t = 0; t < Q::C; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
};

// A step's rows into the state.  MASKED: only the rows before `lim` of columns that take part (`on`); the others' state stays as it is, also
// where a row that they do not see holds NaN.
template <int D, bool F16, bool FP4, bool MASKED>
__device__ __forceinline__ void accumulate(State<D, F16, FP4> &st, const Rows<D, F16, FP4> &f, const f32x4 (&products)[Geo<D, F16, FP4>::kTiles],
                                           float scale_log2, int g, int lim, bool on)
{
    using Q = Geo<D, F16, FP4>;
    float p[4 * Q::kTiles], top = kNone;
#pragma unroll
    for (int t = 0; t < Q::kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x = products[t][i] * scale_log2;
            if (MASKED) x = on && 16 * t + 4 * g + i < lim ? x : -INFINITY;
            p[4 * t + i] = x;
            top = fmaxf(top, x);
        }
    auto larger = [](float a, float b) { return fmaxf(a, b); };
    top = swap_reduce<16>(top, larger);
    top = swap_reduce<32>(top, larger);
    if (__any(top > st.m)) {                                               // seldom after a unit's first steps
        const float m = fmaxf(top, st.m), f0 = __builtin_amdgcn_exp2f(st.m - m);
        st.m = m;
        st.l *= f0;
#pragma unroll
        for (int t = 0; t < Q::C; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) st.o[t][i] *= f0;
    }
    const float base = Q::kShift - st.m;
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * Q::kTiles; ++i) {
        p[i] = __builtin_amdgcn_exp2f(p[i] + base);
        l += p[i];
    }
    st.l += l;
#pragma unroll
    for (int h = 0; h < Q::kTiles / 2; ++h) {
        // the 32 rows of tiles 2 h and 2 h + 1: words of two rows' weights, a piece at a time
        u32x4 w[Q::kPieces];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float a = p[8 * h + 2 * j], b = p[8 * h + 2 * j + 1];
            if constexpr (Q::kHalfP) {
                const f16x2 hi = {(_Float16)a, (_Float16)b};
                w[0][j] = __builtin_bit_cast(uint32_t, hi);
                w[1][j] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)(a - (float)hi.x), (_Float16)(b - (float)hi.y)});
            } else {
#pragma unroll
                for (int k = 0; k < 3; ++k) {                              // cut off, not rounded: three times eight bits are all 24
                    w[k][j] = high_halves(__float_as_uint(a), __float_as_uint(b));
                    a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
                    b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
                }
            }
        }
        float scale[8];
        if constexpr (FP4) {
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                scale[r] = scale_value(f.vs[2 * h + r / 4] >> (8 * (r % 4)) & 255u);
                if (MASKED) scale[r] = 32 * h + 16 * (r / 4) + 4 * g + r % 4 < lim ? scale[r] : 1.f;
            }
        }
#pragma unroll
        for (int k = 0; k < Q::C / 2; ++k) {
            uint32_t x[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const int t = 2 * h + r / 4, i = r % 4;
                if constexpr (FP4) {
                    const int at = i * (Q::C / 2) + k;
                    x[r] = two_codes(f.v[t][at / 4], scale[r], at % 4);
                } else {
                    x[r] = f.v[t][i * (Q::C / 2) + k];
                    if (MASKED) x[r] = 16 * t + 4 * g + i < lim ? x[r] : 0u;
                }
            }
            const u32x4 lo = {low_halves(x[0], x[1]), low_halves(x[2], x[3]), low_halves(x[4], x[5]), low_halves(x[6], x[7])};
            const u32x4 hi = {high_halves(x[0], x[1]), high_halves(x[2], x[3]), high_halves(x[4], x[5]), high_halves(x[6], x[7])};
            f32x4 a = st.o[2 * k], b = st.o[2 * k + 1];
#pragma unroll
            for (int c = Q::kPieces - 1; c >= 0; --c) {
                a = product<Q::kHalfP>(lo, w[c], a);
                b = product<Q::kHalfP>(hi, w[c], b);
            }
            if (MASKED) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    a[i] = on ? a[i] : st.o[2 * k][i];
                    b[i] = on ? b[i] : st.o[2 * k + 1][i];
                }
            }
            st.o[2 * k] = a;
            st.o[2 * k + 1] = b;
        }
    }
}

// grid: (stretches / kWaves, groups of 16 columns)
template <int D, bool F16, bool FP4> __global__ __launch_bounds__(kThreads, 2) void pages_attend_kernel(const AttendArgs a)
{
    using Q = Geo<D, F16, FP4>;
    constexpr int kBytes = FP4 ? Fp4Page<D>::kBytes : WidePage<D>::kBytes;
    __shared__ uint32_t wsum[kWaves];
    __shared__ int start_unit[kWaves];
    __shared__ uint32_t start_at[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    auto steps_of = [&](int u) { return (uint32_t)(clamp_len(a.lens[u], a.max_pages) + Q::kStep - 1) / Q::kStep; };
    // ---- where this wavefront's stretch begins ----
    const int per = (a.n_units + kThreads - 1) / kThreads, u0 = min(tid * per, a.n_units), u1 = min(u0 + per, a.n_units);
    uint32_t mine = 0u;
    for (int u = u0; u < u1; ++u) mine += steps_of(u);
    uint32_t before = wave_prefix_sum(mine) - mine;
    if (lane == 63) wsum[w] = before + mine;
    __syncthreads();
    uint32_t total = 0u;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        before += i < w ? wsum[i] : 0u;
        total += wsum[i];
    }
    const uint32_t stretches = gridDim.x * kWaves, run = max(1u, (total + stretches - 1) / stretches);
    const bool plans = blockIdx.x == 0 && blockIdx.y == 0;
    if (plans || (before < (blockIdx.x + 1) * kWaves * run && before + mine > blockIdx.x * kWaves * run)) {
        uint32_t at = before;
        for (int u = u0; u < u1; ++u) {
            const uint32_t c = steps_of(u);
            if (plans) a.plan[u] = c ? make_int2((int)(at / run) + u, (int)((at + c - 1) / run) + u + 1) : make_int2(0, 0);
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                const uint32_t lo = (blockIdx.x * kWaves + i) * run;
                if (at <= lo && lo < at + c) {
                    start_unit[i] = u;
                    start_at[i] = at;
                }
            }
            at += c;
        }
    }
    __syncthreads();
    const uint32_t stretch = blockIdx.x * kWaves + w, lo = stretch * run, hi = min(lo + run, total);
    if (lo >= hi) return;
    int u = __builtin_amdgcn_readfirstlane(start_unit[w]);
    uint32_t step = lo - __builtin_amdgcn_readfirstlane(start_at[w]);     // of the unit
    // ---- columns ----
    const int cols = a.n_new * a.G, col0 = blockIdx.y * kCols, col = col0 + n;
    const bool there = col < cols;
    const int token = (there ? col : cols - 1) / a.G, head = (there ? col : cols - 1) - token * a.G;
    const int token0 = col0 / a.G, token1 = min(col0 + kCols, cols) - 1 >= 0 ? (min(col0 + kCols, cols) - 1) / a.G : 0;

    Query<D, F16, FP4> q;
    State<D, F16, FP4> st;
    auto begin = [&]() {
        const int s = u / a.H, h = u - s * a.H;
        load_query<D, F16, FP4>(q, a.q + (((int64_t)s * a.n_new + token) * a.H * a.G + h * a.G + head) * D, there, g);
        st.clear();
    };
    auto finish = [&]() {
        float l = st.l;
        auto sum = [](float x, float y) { return x + y; };
        l = swap_reduce<16>(l, sum);
        l = swap_reduce<32>(l, sum);
        if (!there) return;
        float *dst = a.part + (((int64_t)stretch + u) * cols + col) * (D + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * g + i < Q::VL)
#pragma unroll
                for (int t = 0; t < Q::C; t += 4)
                    *reinterpret_cast<f32x4 *>(dst + (4 * g + i) * Q::C + t) = f32x4{st.o[t][i], st.o[t + 1][i], st.o[t + 2][i], st.o[t + 3][i]};
        if (g == 0) {
            dst[D] = st.m - Q::kShift;
            dst[D + 1] = l;
        }
    };
    begin();
    int len = clamp_len(a.lens[u], a.max_pages);
    for (uint32_t i = lo; i < hi; ++i) {
        const int id = a.table[(int64_t)u * a.max_pages + step * Q::kStep / kRows];
        if (id >= 0 && id < a.n_pages) {
            Rows<D, F16, FP4> f;
            load_rows<D, F16, FP4>(f, a.pool + (int64_t)id * kBytes, (int)(step % (kRows / Q::kStep)), n, g);
            f32x4 s[Q::kTiles];
            key_products<D, F16, FP4>(f, q, s);
            const int rel = len - (int)(step * Q::kStep);                  // rows of the step, and behind it
            if (rel - (a.n_new - 1) >= Q::kStep) accumulate<D, F16, FP4, false>(st, f, s, a.scale_log2, g, 0, true);
            else
                for (int t = token0; t <= token1; ++t)
                    accumulate<D, F16, FP4, true>(st, f, s, a.scale_log2, g, rel - (a.n_new - 1 - t), token == t);
        }
        ++step;
        if (i + 1 == hi || (int)(step * Q::kStep) >= len) {
            finish();
            if (i + 1 < hi) {
                do len = clamp_len(a.lens[++u], a.max_pages);
                while (len == 0 && u + 1 < a.n_units);
                step = 0;
                begin();
            }
        }
    }
}

// grid: a workgroup for every unit and column; 256 / D slices of a unit's parts, added up in the slices' order
template <int D> __global__ __launch_bounds__(256) void pages_combine_kernel(const float *__restrict__ part, const int2 *__restrict__ plan, int cols,
                                                                             int H, int G, int n_new, float *__restrict__ out, float *__restrict__ lse)
{
    constexpr int NS = 256 / D, U = 4;
    __shared__ float red[4], lds_l[NS], lds_o[NS][D];
    const int u = blockIdx.x / cols, col = blockIdx.x - u * cols, tid = threadIdx.x, e = tid % D, sl = tid / D;
    const int2 of = plan[u];
    const float *src = part + (int64_t)col * (D + 4);
    const int64_t each = (int64_t)cols * (D + 4);
    float mm = kNone, ll = 0.f, oo = 0.f;
    for (int i = of.x + tid; i < of.y; i += 256) mm = fmaxf(mm, src[i * each + D]);
    mm = wave_max(mm);
    if ((tid & 63) == 0) red[tid >> 6] = mm;
    __syncthreads();
    mm = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    if (sl < NS) {
        for (int i = of.x + sl; i < of.y; i += U * NS) {
            float pm[U], pl[U], po[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const float *p = src + min(i + k * NS, of.y - 1) * each;
                pm[k] = p[D], pl[k] = p[D + 1], po[k] = p[e];
            }
#pragma unroll
            for (int k = 0; k < U; ++k)
                if (i + k * NS < of.y) {
                    const float f = __builtin_amdgcn_exp2f(pm[k] - mm);
                    ll = fmaf(f, pl[k], ll);
                    oo = fmaf(f, po[k], oo);
                }
        }
        lds_o[sl][e] = oo;
        if (e == 0) lds_l[sl] = ll;
    }
    __syncthreads();
    if (sl > 0) return;
    for (int i = 1; i < NS; ++i) {
        oo += lds_o[i][e];
        ll += lds_l[i];
    }
    const int s = u / H, h = u - s * H, t = col / G, g = col - t * G;
    const int64_t row = ((int64_t)s * n_new + t) * H * G + h * G + g;
    const bool none = ll == 0.f;                                           // (NaN is handed on)
    out[row * D + e] = none ? 0.f : oo / ll;
    if (lse && e == 0) lse[row] = none ? -INFINITY : (mm + log2f(ll)) * kLn2;
}

int step_rows(int format) { return format == NKV_PAGES_FP4 ? 64 : 32; }
unsigned groups_of(const nkv_pages &p)
{
    const int64_t most = (int64_t)p.n_seqs * p.H * p.max_pages * (kRows / step_rows(p.format));
    return (unsigned)std::min<int64_t>(kMostGroups, (most + kWaves - 1) / kWaves);
}
size_t plan_bytes(const nkv_pages &p) { return ((size_t)p.n_seqs * p.H * sizeof(int2) + 255) / 256 * 256; }

}  // namespace

size_t pages_ws_bytes(const nkv_pages &p, int n_q_heads, int n_new)
{
    const size_t cols = (size_t)(n_q_heads / p.H) * n_new;
    return plan_bytes(p) + ((size_t)groups_of(p) * kWaves + (size_t)p.n_seqs * p.H) * cols * (p.d + 4) * sizeof(float);
}

hipError_t launch_pages_attention(const void *q, const nkv_pages &p, int n_q_heads, int n_new, double scale, float *out, float *lse, void *ws,
                                  hipStream_t st)
{
    AttendArgs a{};
    a.q = (const uint16_t *)q, a.pool = (const uint8_t *)p.pool, a.table = p.table, a.lens = p.lens;
    a.n_units = p.n_seqs * p.H, a.H = p.H, a.G = n_q_heads / p.H, a.n_new = n_new, a.n_pages = p.n_pages, a.max_pages = p.max_pages;
    a.scale_log2 = (float)(scale * 1.4426950408889634);
    a.plan = (int2 *)ws;
    a.part = (float *)((char *)ws + plan_bytes(p));
    const int cols = a.G * n_new;
    const dim3 grid(groups_of(p), (unsigned)((cols + kCols - 1) / kCols));
    for_head_dim(p.d, [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        const bool f16 = p.dtype == NKV_DTYPE_F16, fp4 = p.format == NKV_PAGES_FP4;
        (f16 ? fp4 ? pages_attend_kernel<D, true, true> : pages_attend_kernel<D, true, false>
             : fp4 ? pages_attend_kernel<D, false, true> : pages_attend_kernel<D, false, false>)<<<grid, kThreads, 0, st>>>(a);
        pages_combine_kernel<D><<<(unsigned)(a.n_units * cols), 256, 0, st>>>(a.part, a.plan, cols, a.H, a.G, n_new, out, lse);
    });
    return hipGetLastError();
}

}  // namespace nkv
