// Rows into and out of the paged cache: new tokens, rotated on the way (nkv_pages_append), and the packed rows that the
// compression operator leaves (nkv_pages_load, nkv_pages_read).
//
// All three move each byte once and compute little: 16-byte loads, one thread for eight dims of a row.  A block of the 4-bit format is
// 32 dims, so four neighbouring lanes find its scale among themselves.
#include "nkv_pages.h"

#include <algorithm>

namespace nkv {
namespace {

__device__ __forceinline__ int64_t clamp_row(int64_t r, int64_t rows) { return r < 0 ? 0 : (r > rows ? rows : r); }
__device__ __forceinline__ int clamp_len(int len, int max_pages) { return max(0, min(len, max_pages * kRows)); }

// Dims 8 c .. 8 c + 7 of one row as fp32 into the page's rows of K (or V), in the cache's form.  Lanes 4 i .. 4 i + 3 hold a block.
// (w: the same in 16 bits, for pages that hold those)
template <int D, bool F16, bool FP4> __device__ __forceinline__ void store_row(uint8_t *page, bool key, int row, int c, const float (&x)[8], const u32x4 &w16)
{
    if constexpr (FP4) {
        using P = Fp4Page<D>;
        const uint32_t scale = fp4_scale(x), w = fp4_codes(x, scale);
        if (key) *reinterpret_cast<uint32_t *>(page + P::k_code(row, 8 * c)) = w;
        else store_v_codes<D>(page, row, c, w);
        if (c % 4 == 0) page[key ? P::k_scale(row, c / 4) : P::v_scale(row, c / 4)] = (uint8_t)scale;
    } else {
        using P = WidePage<D>;
        *reinterpret_cast<u32x4 *>(page + (key ? P::k(row, 8 * c) : P::v(row, 8 * c))) = w16;
    }
}

// To 32 bits, and not on to 16 in one rounding: the compiler would make one of two.
__device__ __forceinline__ float rounded(double x)
{
    float f = (float)x;
    asm volatile("" : "+v"(f));
    return f;
}

struct AppendArgs {
    const void *k, *v, *q;
    void *q_out;
    int64_t k_str[3], v_str[3], q_str[3];
    const int32_t *positions;
    const float *rope;
    int32_t n_new, Hq, rot, halves, n_positions, H, n_pages, max_pages;
    const int32_t *table, *lens;
    uint8_t *pool;
};

// A token's row in `slot`, 16 bytes from dim d0 and from d1 on, and where it goes: row and page of its unit.  (Everything by value: captured pointers that a lane
// chooses among would lie in memory.)
struct Slot {
    u32x4 a, b;
    int row, page;
};
__device__ __forceinline__ Slot load_slot(int slot, const uint16_t *kb, const uint16_t *vb, const uint16_t *qb, int64_t kh, int64_t vh, int64_t qh, int H,
                                          int d0, int d1, const int32_t *lens, const int32_t *table, int max_pages, int behind)
{
    const bool key = slot < H, value = !key && slot < 2 * H;
    const int h = key ? slot : value ? slot - H : slot - 2 * H;
    const uint16_t *src = (key ? kb : value ? vb : qb) + h * (key ? kh : value ? vh : qh);
    Slot s{*reinterpret_cast<const u32x4 *>(src + d0), *reinterpret_cast<const u32x4 *>(src + d1), 0, -1};
    if (key || value) {
        s.row = clamp_len(lens[h], max_pages) + behind;
        if (s.row >= 0) s.page = table[(int64_t)h * max_pages + s.row / kRows];
    }
    return s;
}

// A workgroup for a token's heads (K heads, V heads, query heads), or a share of them: kRowsAt rows at a time.  A thread keeps its dims' cosines and sines for
// all of its rows, and takes eight dims of a row, or, BOTH, two times eight: both dims of eight pairs (or eight and eight that are not rotated), so that each is
// read and widened once.  In 64 bits the products of a 16-bit value and a 24-bit cosine are exact, so the result is one rounding of the sum, then one to 32 bits,
// whatever the order of the operations.  3 x 2731 tokens of 8 + 32 heads, head dim 128: eight dims a thread 46.6 us, twice eight 36.9 to 37.9 (4.8 TB/s), with the next
// rows asked for before a row is worked on 41.8: it is wavefronts, and their instructions, half of them in 64 bits, that it takes, not loads in flight.
template <int D, bool F16, bool FP4, bool BOTH> __global__ __launch_bounds__(256) void append_kernel(const AppendArgs a)
{
    constexpr int CPR = D / 8, kLanes = BOTH ? CPR / 2 : CPR, kRowsAt = 256 / kLanes;
    const int r = threadIdx.x / kLanes, c = threadIdx.x % kLanes, tok = blockIdx.x, s = tok / a.n_new, t = tok - s * a.n_new, slots = 2 * a.H + a.Hq;
    if (r >= kRowsAt) return;
    const int half = a.rot / 2;
    // the thread's dims from d0, and, BOTH, from d1 on; else d1 is the partner of d0
    bool turns = 8 * c < (BOTH ? half : a.rot), first = true;
    int d0 = 8 * c, d1 = 8 * c + half;
    if (BOTH) {
        if (!turns) d0 += half, d1 = d0 + D / 2 - half;
    } else {
        first = 8 * c < half;
        d1 = !turns || !a.halves ? d0 : first ? d0 + half : d0 - half;
    }
    const int step = gridDim.y * kRowsAt, slot0 = blockIdx.y * kRowsAt + r;
    const uint16_t *kb = (const uint16_t *)a.k + s * a.k_str[0] + t * a.k_str[1], *vb = (const uint16_t *)a.v + s * a.v_str[0] + t * a.v_str[1],
                   *qb = (const uint16_t *)a.q + s * a.q_str[0] + t * a.q_str[1];
    const int64_t kh = a.k_str[2], vh = a.v_str[2], qh = a.q_str[2];
    const int32_t *lens = a.lens + (int64_t)s * a.H, *table = a.table + (int64_t)s * a.H * a.max_pages;
    const int pos = a.positions ? a.positions[tok] : 0;
    if (pos < 0 || (a.rot > 0 && pos >= a.n_positions)) return;
    double co[8], si[8];
    if (turns) {
        const float *cs = a.rope + (int64_t)pos * a.rot, *sn = cs + half;
        if (BOTH || a.halves) {
            const int e = first ? 8 * c : 8 * c - half;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                co[k] = cs[e + k];
                si[k] = first ? -sn[e + k] : sn[e + k];
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                co[k] = co[k + 1] = cs[4 * c + k / 2];
                si[k + 1] = sn[4 * c + k / 2];
                si[k] = -si[k + 1];
            }
        }
    }
    auto put = [&](int slot, int page_id, int page_row, int dim, const float (&x)[8], const u32x4 &w) {
        if (slot >= 2 * a.H) *reinterpret_cast<u32x4 *>((uint16_t *)a.q_out + ((int64_t)tok * a.Hq + slot - 2 * a.H) * D + dim) = w;
        else if (page_id >= 0 && page_id < a.n_pages)
            store_row<D, F16, FP4>(a.pool + (int64_t)page_id * (FP4 ? Fp4Page<D>::kBytes : WidePage<D>::kBytes), slot < a.H, page_row & (kRows - 1), dim / 8, x, w);
    };
    for (int slot = slot0; slot < slots; slot += step) {
        const Slot at = load_slot(slot, kb, vb, qb, kh, vh, qh, a.H, d0, d1, lens, table, a.max_pages, t - a.n_new);
        const bool rotated = turns && (slot < a.H || slot >= 2 * a.H);
        u32x4 w = at.a, v = at.b;
        float x[8], y[8];
        unpack8<F16>(w, x);
        unpack8<F16>(v, y);
        if (rotated) {
            if constexpr (BOTH) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const double p = x[k], q = y[k];
                    x[k] = rounded(fma(p, co[k], q * si[k]));
                    y[k] = rounded(fma(q, co[k], p * -si[k]));
                }
                v = pack8<F16>(y);
            } else {
                if (!a.halves)
#pragma unroll
                    for (int k = 0; k < 8; k += 2) y[k] = x[k + 1], y[k + 1] = x[k];
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = rounded(fma((double)x[k], co[k], (double)y[k] * si[k]));
            }
            w = pack8<F16>(x);
        }
        put(slot, at.page, at.row, d0, x, w);
        if (BOTH) put(slot, at.page, at.row, d1, y, v);
    }
}

// The unit that number i belongs to: its packed rows off .. off + n - 1, its length, and its first number.
struct Span {
    int unit, len;
    int64_t off, n, number;
};
__device__ __forceinline__ int64_t of_lane(int64_t x, int lane)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)x >> 32), lane);
    return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ Span span_of(const int64_t *head_off, const int32_t *lens, int n_units, int64_t rows, int max_pages, int64_t i)
{
    Span s;
    if (n_units <= kWave) {                                                // everything that may be asked for at once
        const int lane = threadIdx.x & (kWave - 1), u = min(lane, n_units - 1);
        const int64_t from = clamp_row(head_off[u], rows), to = clamp_row(head_off[u + 1], rows);
        const int len = lens[u];
        const int64_t number = lane == 0 ? 0 : from / kRows + 2 * (int64_t)lane;
        s.unit = 63 - __builtin_clzll(__ballot(lane < n_units && number <= i));   // (lane 0 is always among them)
        s.off = of_lane(from, s.unit), s.n = of_lane(to, s.unit) - s.off, s.number = of_lane(number, s.unit);
        s.len = clamp_len(__builtin_amdgcn_readlane(len, s.unit), max_pages);
    } else {
        s.unit = __builtin_amdgcn_readfirstlane(
            wave_search_fn(n_units, i, [&](int x) { return x == 0 ? (int64_t)0 : clamp_row(head_off[x], rows) / kRows + 2 * (int64_t)x; }));
        s.off = clamp_row(head_off[s.unit], rows), s.n = clamp_row(head_off[s.unit + 1], rows) - s.off;
        s.number = s.unit == 0 ? 0 : s.off / kRows + 2 * (int64_t)s.unit;
        s.len = clamp_len(lens[s.unit], max_pages);
    }
    return s;
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
    const Span sp = span_of(head_off, lens, n_units, rows, max_pages, i);
    const int u = sp.unit, len = sp.len;
    const int64_t first = len - sp.n;                                     // of the unit's rows, the one that the first packed one is
    const int64_t j = (first >= 0 ? first / kRows : -((-first + kRows - 1) / kRows)) + i - sp.number;
    if (sp.n <= 0 || j * kRows >= len) return;
    const int id = j >= 0 ? table[(int64_t)u * max_pages + j] : -1;
    const bool there = id >= 0 && id < n_pages;
    if (LOAD && !there) return;
    uint8_t *page = pool + (there ? (int64_t)id : 0) * (FP4 ? Fp4Page<D>::kBytes : WidePage<D>::kBytes);
    const int c = threadIdx.x % CPR, r = threadIdx.x / CPR;
    const int64_t at0 = sp.off + j * kRows - first;                       // packed row of the page's row 0
    const int lo = (int)max(first - j * kRows, (int64_t)0), hi = (int)min(len - j * kRows, (int64_t)kRows);   // the page's rows
    if constexpr (LOAD || !FP4) {
        u32x4 w[2][4];                                                    // (rows outside: others' that are asked for anyway)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int row = min(max(16 * t + r, lo), hi - 1);
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                if constexpr (LOAD) w[kv][t] = __builtin_nontemporal_load(reinterpret_cast<u32x4 *>((kv == 0 ? pk : pv) + (at0 + row) * D + 8 * c));
                else w[kv][t] = *reinterpret_cast<const u32x4 *>(page + (kv == 0 ? WidePage<D>::k(row, 8 * c) : WidePage<D>::v(row, 8 * c)));
            }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int row = 16 * t + r;
            if (row < lo || row >= hi) continue;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                if constexpr (LOAD) {
                    float x[8];
                    unpack8<F16>(w[kv][t], x);
                    store_row<D, F16, FP4>(page, kv == 0, row, c, x, w[kv][t]);
                } else {
                    __builtin_nontemporal_store(there ? w[kv][t] : u32x4{0u, 0u, 0u, 0u}, reinterpret_cast<u32x4 *>((kv == 0 ? pk : pv) + (at0 + row) * D + 8 * c));
                }
            }
        }
    } else {
        // all of the page's codes and scales first: a row's scales lie with those of the rows 16, 32 and 48 further on
        using P = Fp4Page<D>;
        uint32_t code[2][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            code[0][t] = *reinterpret_cast<const uint32_t *>(page + P::k_code(16 * t + r, 8 * c));
            code[1][t] = load_v_codes<D>(page, 16 * t + r, c);
        }
        const uint32_t ks = *reinterpret_cast<const uint32_t *>(page + P::k_scale(r, c / 4));
        const u32x4 vs = *reinterpret_cast<const u32x4 *>(page + P::v_scale(r / 4 * 4, c / 4));
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int row = 16 * t + r;
            if (row < lo || row >= hi) continue;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                u32x4 w = fp4_rows<F16>(code[kv][t], kv == 0 ? ks >> (8 * t) & 255u : vs[t] >> (8 * (r % 4)) & 255u);
                if (!there) w = u32x4{0u, 0u, 0u, 0u};
                __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>((kv == 0 ? pk : pv) + (at0 + row) * D + 8 * c));
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
    const int64_t tokens = (int64_t)p.n_seqs * t.n_new;
    // Both dims of a pair in a thread; in 4 bits where the four threads of a block still lie side by side.  (3 x 2731 tokens of 8 + 32 heads, 16 bits, 32 of 128 dims
    // rotated: 39.9 us, and 42.9 with eight dims a thread.  Neighbouring dims as pairs, or no rotation: eight a thread 37.6 and 34.6 us, sixteen 39.3 and
    // 35.8.  Neighbours at head dim 96, 5 x 389 tokens of 32 + 32 heads, fp16 in 4 bits: eight 17.2, sixteen 16.0.  Eight for all neighbours, one kernel less: what
    // sixteen gain there is less than what they lose at 128.)
    const bool both = t.rot > 0 && a.halves && (p.format != NKV_PAGES_FP4 || (t.rot % 64 == 0 && p.d % 64 == 0));
    // Tokens enough to fill the chip: a workgroup takes all of a token's heads, and loads its angles once; fewer: a share of them.
    const int at_once = 256 / (p.d / (both ? 16 : 8)), most = (2 * p.H + t.n_q_heads + at_once - 1) / at_once;
    const dim3 groups((unsigned)tokens, (unsigned)std::max<int64_t>(1, std::min<int64_t>(most, 2048 / tokens)));
    for_head_dim(p.d, [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        auto go = [&](auto f16, auto fp4) {
            constexpr bool F16 = decltype(f16)::value, FP4 = decltype(fp4)::value;
            if constexpr (!FP4 || D % 64 == 0) {
                if (both) return append_kernel<D, F16, FP4, true><<<groups, 256, 0, st>>>(a);
            }
            append_kernel<D, F16, FP4, false><<<groups, 256, 0, st>>>(a);
        };
        using Yes = std::true_type;
        using No = std::false_type;
        const bool f16 = p.dtype == NKV_DTYPE_F16, fp4 = p.format == NKV_PAGES_FP4;
        if (f16 && fp4) go(Yes{}, Yes{});
        else if (f16) go(Yes{}, No{});
        else if (fp4) go(No{}, Yes{});
        else go(No{}, No{});
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
