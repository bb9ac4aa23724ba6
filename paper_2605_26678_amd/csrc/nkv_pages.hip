// Rows into and out of the paged cache: new tokens, rotated on the way (nkv_pages_append), and the packed rows that the
// compression operator leaves (nkv_pages_load, nkv_pages_read).
//
// All three move each byte once and compute little: 16-byte loads, one thread for eight dims of a row.  A block of the 4-bit format is
// 32 dims, so four neighbouring lanes find its scale among themselves.
#include "nkv_pages.h"

namespace nkv {
namespace {

__device__ __forceinline__ int64_t clamp_row(int64_t r, int64_t rows) { return r < 0 ? 0 : (r > rows ? rows : r); }
__device__ __forceinline__ int clamp_len(int len, int max_pages) { return max(0, min(len, max_pages * kRows)); }

// Dims 8 c .. 8 c + 7 of one row as fp32 into the page's rows of K (or V), in the cache's form.  Lanes 4 i .. 4 i + 3 hold a block.
template <int D, bool F16, bool FP4> __device__ __forceinline__ void store_row(uint8_t *page, bool key, int row, int c, const float (&x)[8])
{
    if constexpr (FP4) {
        using P = Fp4Page<D>;
        const uint32_t scale = fp4_scale(x), w = fp4_codes(x, scale);
        if (key) *reinterpret_cast<uint32_t *>(page + P::k_code(row, 8 * c)) = w;
        else store_v_codes<D>(page, row, c, w);
        if (c % 4 == 0) page[key ? P::k_scale(row, c / 4) : P::v_scale(row, c / 4)] = (uint8_t)scale;
    } else {
        using P = WidePage<D>;
        *reinterpret_cast<u32x4 *>(page + (key ? P::k(row, 8 * c) : P::v(row, 8 * c))) = pack8<F16>(x);
    }
}

struct AppendArgs {
    const void *k, *v, *q;
    void *q_out;
    int64_t k_str[3], v_str[3], q_str[3];
    const int32_t *positions;
    const float *rope;
    int32_t n_new, Hq, rot, halves, n_positions, H, n_pages, max_pages;
    uint32_t threads;
    const int32_t *table, *lens;
    uint8_t *pool;
};

// A thread for 16 bytes of k, v or q, in the order of a token's heads: K heads, V heads, query heads.  The rotation's partner of a dim
// is read by both threads of the pair (from the caches), so no thread waits for another.  In 64 bits the products of a 16-bit value and a
// 24-bit cosine are exact, so the result is one rounding of the sum, then one to 32 bits, whatever the order of the operations.
template <int D, bool F16, bool FP4> __global__ __launch_bounds__(256) void append_kernel(const AppendArgs a)
{
    constexpr uint32_t CPR = D / 8;
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    if (i >= a.threads) return;                                            // (whole rows)
    const uint32_t item = i / CPR, slots = 2u * a.H + a.Hq, tok = item / slots, slot = item - tok * slots;
    const int c = (int)(i - item * CPR), s = (int)(tok / (uint32_t)a.n_new), t = (int)(tok - (uint32_t)s * a.n_new);
    const bool key = slot < (uint32_t)a.H, value = !key && slot < 2u * a.H;
    const int h = key ? slot : value ? slot - a.H : slot - 2 * a.H;
    const int pos = a.positions ? a.positions[tok] : 0;
    if (pos < 0 || (a.rot > 0 && pos >= a.n_positions)) return;
    int row = 0;
    uint8_t *page = nullptr;
    if (key || value) {
        const int u = s * a.H + h;
        row = clamp_len(a.lens[u], a.max_pages) - a.n_new + t;
        if (row < 0) return;
        const int id = a.table[(int64_t)u * a.max_pages + row / kRows];
        if (id < 0 || id >= a.n_pages) return;
        page = a.pool + (int64_t)id * (FP4 ? Fp4Page<D>::kBytes : WidePage<D>::kBytes);
    }
    const int64_t *str = key ? a.k_str : value ? a.v_str : a.q_str;
    const uint16_t *src = (const uint16_t *)(key ? a.k : value ? a.v : a.q) + s * str[0] + t * str[1] + h * str[2];
    float x[8];
    unpack8<F16>(*reinterpret_cast<const u32x4 *>(src + 8 * c), x);
    if (!value && 8 * c < a.rot) {
        const int half = a.rot / 2;
        const float *cs = a.rope + (int64_t)pos * a.rot, *sn = cs + half;
        if (a.halves) {
            const bool first = 8 * c < half;
            const int e = first ? 8 * c : 8 * c - half;
            float y[8];
            unpack8<F16>(*reinterpret_cast<const u32x4 *>(src + (first ? 8 * c + half : e)), y);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const double m = (double)y[k] * (double)sn[e + k];
                x[k] = (float)fma((double)x[k], (double)cs[e + k], first ? -m : m);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const double co = cs[4 * c + k / 2], si = sn[4 * c + k / 2], p = x[k], r = x[k + 1];
                x[k] = (float)fma(p, co, -(r * si));
                x[k + 1] = (float)fma(r, co, p * si);
            }
        }
    }
    if (key || value) store_row<D, F16, FP4>(page, key, row & (kRows - 1), c, x);
    else *reinterpret_cast<u32x4 *>((uint16_t *)a.q_out + ((int64_t)tok * a.Hq + h) * D + 8 * c) = pack8<F16>(x);
}

// Packed rows to and from the pages.  A workgroup takes one page of one unit: 16 rows at a time, D / 8 threads a row.  The pages that a unit's
// rows touch are numbered from off[u] / 64 + 2 u on, which leaves room for all of them (n rows touch at most n / 64 + 2 pages), so no kernel plans in front.
// grid: as many numbers as there are.
template <int D, bool F16, bool FP4, bool LOAD>
__global__ __launch_bounds__(2 * D) void rows_kernel(uint16_t *__restrict__ pk, uint16_t *__restrict__ pv, const int64_t *__restrict__ head_off,
                                                    int64_t rows, int n_units, uint8_t *__restrict__ pool, const int32_t *__restrict__ table,
                                                    const int32_t *__restrict__ lens, int n_pages, int max_pages)
{
    constexpr int CPR = D / 8;
    const int64_t i = blockIdx.x;
    const int u = __builtin_amdgcn_readfirstlane(
        wave_search_fn(n_units, i, [&](int x) { return x == 0 ? (int64_t)0 : clamp_row(head_off[x], rows) / kRows + 2 * (int64_t)x; }));
    const int64_t off = clamp_row(head_off[u], rows), n = clamp_row(head_off[u + 1], rows) - off;
    const int len = clamp_len(lens[u], max_pages);
    const int64_t first = len - n;                                        // of the unit's rows, the one that `off` is
    const int64_t j = (first >= 0 ? first / kRows : -((-first + kRows - 1) / kRows)) + i - (u == 0 ? 0 : off / kRows + 2 * (int64_t)u);
    if (n <= 0 || j * kRows >= len) return;
    const int id = j >= 0 ? table[(int64_t)u * max_pages + j] : -1;
    const bool there = id >= 0 && id < n_pages;
    if (LOAD && !there) return;
    uint8_t *page = pool + (there ? (int64_t)id : 0) * (FP4 ? Fp4Page<D>::kBytes : WidePage<D>::kBytes);
    const int c = threadIdx.x % CPR, r = threadIdx.x / CPR;
    const int64_t at0 = off + j * kRows - first;                          // packed row of the page's row 0
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int row = 16 * t + r;
        const int64_t unit_row = j * kRows + row, at = (at0 + row) * D + 8 * c;
        if (unit_row < first || unit_row >= len) continue;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            u32x4 *rowp = reinterpret_cast<u32x4 *>((kv == 0 ? pk : pv) + at);
            if constexpr (LOAD) {
                if constexpr (FP4) {
                    float x[8];
                    unpack8<F16>(__builtin_nontemporal_load(rowp), x);
                    store_row<D, F16, true>(page, kv == 0, row, c, x);
                } else {
                    *reinterpret_cast<u32x4 *>(page + (kv == 0 ? WidePage<D>::k(row, 8 * c) : WidePage<D>::v(row, 8 * c))) = __builtin_nontemporal_load(rowp);
                }
            } else {
                u32x4 w = {0u, 0u, 0u, 0u};
                if (there) {
                    if constexpr (FP4) {
                        using P = Fp4Page<D>;
                        float x[8];
                        fp4_values(kv == 0 ? *reinterpret_cast<const uint32_t *>(page + P::k_code(row, 8 * c)) : load_v_codes<D>(page, row, c),
                                   page[kv == 0 ? P::k_scale(row, c / 4) : P::v_scale(row, c / 4)], x);
                        constexpr float top = F16 ? 65504.f : 0x1.fep127f;
#pragma unroll
                        for (int k = 0; k < 8; ++k) x[k] = x[k] > top ? top : x[k] < -top ? -top : x[k];
                        w = pack8<F16>(x);
                    } else {
                        w = *reinterpret_cast<const u32x4 *>(page + (kv == 0 ? WidePage<D>::k(row, 8 * c) : WidePage<D>::v(row, 8 * c)));
                    }
                }
                __builtin_nontemporal_store(w, rowp);
            }
        }
    }
}

}  // namespace

bool pages_row_supported(int dtype, int d)
{
    return (dtype == NKV_DTYPE_BF16 || dtype == NKV_DTYPE_F16) && for_head_dim(d, [](auto) {});
}

hipError_t launch_pages_append(const nkv_tokens &t, const nkv_pages &p, hipStream_t st)
{
    AppendArgs a{};
    a.k = t.k, a.v = t.v, a.q = t.q, a.q_out = t.q_out;
    for (int i = 0; i < 3; ++i) a.k_str[i] = t.k_strides[i], a.v_str[i] = t.v_strides[i], a.q_str[i] = t.q_strides[i];
    a.positions = t.positions, a.rope = t.rope;
    a.n_new = t.n_new, a.Hq = t.n_q_heads, a.rot = t.rot, a.halves = t.rope_style == NKV_ROPE_HALVES, a.n_positions = t.n_positions;
    a.H = p.H, a.n_pages = p.n_pages, a.max_pages = p.max_pages;
    a.table = p.table, a.lens = p.lens, a.pool = (uint8_t *)p.pool;
    a.threads = (uint32_t)((int64_t)p.n_seqs * t.n_new * (2 * p.H + t.n_q_heads) * (p.d / 8));
    const unsigned groups = (unsigned)(((int64_t)a.threads + 255) / 256);
    for_head_dim(p.d, [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        const bool f16 = p.dtype == NKV_DTYPE_F16, fp4 = p.format == NKV_PAGES_FP4;
        (f16 ? fp4 ? append_kernel<D, true, true> : append_kernel<D, true, false> : fp4 ? append_kernel<D, false, true> : append_kernel<D, false, false>)<<<groups, 256, 0, st>>>(a);
    });
    return hipGetLastError();
}

hipError_t launch_pages_rows(bool load, const void *k, const void *v, const int64_t *head_off, int64_t rows, const nkv_pages &p, hipStream_t st)
{
    if (rows == 0) return hipSuccess;
    const int n_units = p.n_seqs * p.H;
    const unsigned groups = (unsigned)(rows / kRows + 2 * (int64_t)n_units);
    for_head_dim(p.d, [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        auto go = [&](auto f16, auto fp4) {
            constexpr bool F16 = decltype(f16)::value, FP4 = decltype(fp4)::value;
            (load ? rows_kernel<D, F16, FP4, true> : rows_kernel<D, F16, FP4, false>)<<<groups, 2 * D, 0, st>>>(
                (uint16_t *)k, (uint16_t *)v, head_off, rows, n_units, (uint8_t *)p.pool, p.table, p.lens, p.n_pages, p.max_pages);
        };
        using Yes = std::true_type;
        using No = std::false_type;
        if (p.format != NKV_PAGES_FP4) go(No{}, No{});                      // 16-bit rows are copied as they are
        else if (p.dtype == NKV_DTYPE_F16) go(Yes{}, Yes{});
        else go(No{}, Yes{});
    });
    return hipGetLastError();
}

}  // namespace nkv
