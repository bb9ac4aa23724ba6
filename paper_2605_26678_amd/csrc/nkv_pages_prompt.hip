// nkv_pages_prompt_attention: which kernel takes a call.
#include "nkv_pages_prompt.h"

#include <algorithm>
#include <cmath>

namespace nkv {
namespace {

// Tables of up to that many pages: all rows in one launch, and no scratch.  That costs where the tiles are few: 256 rows, us so and shared out in two, 128 columns of a unit of 256 dims
// 26.9 and 21.2, 256 of 128 dims 17.8 and 15.3; 8 units of 256 columns of 128 dims are not shared out by the rule below either (18.1 and 18.1).
constexpr int kShort = 4;

struct Grid {
    int tiles, splits;                   // workgroups of a unit: tiles of columns, and shares of the rows that one sees
};
// Where the tiles are few, the rows are shared out too, up to as many workgroups as the chip holds at once, two pages each at least.  That shortens the walk over the pages, at 0.7 us each
// and 0.8 for products of 256 columns by 128 dims, but every share's weighted values are written and read again, at some 4 TB/s: the sum is least where both are equal.  us, without
// shares, with those and with as many as the chip holds (8 by 4 heads of 128 dims where nothing else is said):
//   512 tokens 24.7, 24.7 (none), 29.2;  100 tokens behind 1000 40, 23.2 (6), 25.2;  256 tokens behind 8192 243, 57.7 (8), 57.7;  twice what it holds 72;  32 heads of 64 dims, 500 tokens
//   15.3, 15.3 (none), 20.6;  2000 tokens, 4 by 2 heads of 64 dims 39.1, 25.4 (4), 26.4;  4000 tokens, 1 by 8 heads of 96 dims 87, 64 (2), 64;  with one workgroup a compute unit 87
Grid grid_of(const nkv_pages &p, int n_q_heads, int n_new)
{
    const bool two = p.dtype == NKV_DTYPE_F16 && p.format == NKV_PAGES_FP4;
    const int64_t cols = (int64_t)(n_q_heads / p.H) * n_new, at_once = 32 * prompt_waves(p.d, two), units = (int64_t)p.n_seqs * p.H;
    const int64_t tiles = (cols + at_once - 1) / at_once, most = std::min<int64_t>(256 * prompt_groups(p.d, two) / (units * tiles), p.max_pages / 2);
    if (p.max_pages <= kShort || most <= 1) return {(int)tiles, 1};
    const double walk = p.max_pages * (0.7 + 0.8 * (two ? 2 : 1) * std::min(cols, at_once) * p.d / 32768.0), part = units * cols * (p.d + 4) * 8 / 4e6;
    const int splits = (int)std::min((double)most, std::max(1.0, std::floor(std::sqrt(walk / part) + 0.5)));
    return {(int)tiles, splits > 1 && walk / splits + splits * part + 2 < walk ? splits : 1};
}

// Whether a call goes with the single tokens' kernels, where no workgroup has a unit to itself (below).  They share out all units' pages evenly and take up to 16 columns at a time, in some
// 10 us and what memory takes; the tiles take a page a microsecond in each workgroup whatever the columns, in one launch or two.  us, theirs / tiles, 8 KV heads of 128 dims:
//   4 bits    16 columns: 16384 rows of 1, 32 sequences 15 / 22, 112 / 363
//             32 columns: 1024 rows 10.6 / 10.8, 37 / 27; 4096 rows 11 / 16, 79 / 90; 16384 rows 23 / 23, 216 / 363
//             64 columns: 4096 rows 13 / 17, 150 / 93;  one column, 3 rows of 33 sequences with 32 heads 14 / 26
//   16 bits   8 columns: 600, 1024 rows of 1 sequence 12.8 / 10.6, 11.9 / 10.3; 1 sequence of up to 1400, 4096, 16384 rows (a quarter to all of them, as units have) 12.7 / 11.3, 13.4 / 12.7, 16.5 / 20.8;
//             4 of 1400, 4096, 16384 13.8 / 11.9, 20.8 / 18.9, 50 / 48; 32 of 16384 246 / 346, and all of the same length 366 / 365
//             32 columns: 4096 rows of 1, 32 sequences 14.5 / 15.7, 246 / 98
// (16 bits, some thousand rows of a few sequences: up to 2 us more than the tiles take.)
bool few_columns(const nkv_pages &p, int n_q_heads, int n_new)
{
    const int64_t cols = (int64_t)(n_q_heads / p.H) * n_new;
    return p.format == NKV_PAGES_FP4 ? cols <= (p.max_pages > 32 ? 32 : 16) : cols <= 16 && p.max_pages > 20;
}

// Whether up to 16 columns have a workgroup a unit, in one launch: where that takes less than two launches' 10 us and what memory takes, by the pages that a unit may have, of which it
// has 0.7 in the mean (the stretches' pages are shared out evenly, a unit's by the workgroup alone).  A workgroup takes a unit's pages at 25 to 34 us a MiB, 4-bit ones 33 to 38, by how many
// others there are; 4 us for the next one on the same compute unit.  us, alone / otherwise, 8 KV heads of 128 dims:
//   4 bits    1 sequence of 250, 500, 1024, 2000 rows 6.9 / 10.3, 7.0 / 10.2, 9.6 / 10.2, 13.3 / 10.4;  32 sequences 7.0 / 13.4, 7.4 / 15.3, 10.7 / 20, 15.3 / 24, of 4000 rows 26.6 / 32.4
//   16 bits   1 sequence 7.7 / 10.9, 10.6 / 10.9, 17.4 / 11.1;  16 sequences 8.5 / 11.1, 13.4 / 14.1, 22.2 / 22.3, of 4000 rows 64.8 / 56.9;  32 9.4 / 11.6, 14.9 / 18.8, 25 / 32, 76 / 100
//   one token of 33 sequences with 32 KV heads, 3 rows each: 21 / 15 (so: 512 units at most)
bool alone(const nkv_pages &p, int n_q_heads, int n_new, int64_t pages, double slack = 1.0)
{
    const int64_t units = (int64_t)p.n_seqs * p.H, cols = (int64_t)(n_q_heads / p.H) * n_new;
    if (cols > 16 || units > 512) return false;
    const bool four = p.format == NKV_PAGES_FP4;
    const double kib = (four ? p.d * 64 + p.d * 4 : p.d * 256) / 1024.0, full = units / 256.0, share = std::min(1.0, full);
    const double page = kib * (four ? 0.033 * (1 + 0.15 * share) : 0.025 + 0.009 * share) * std::max(1.0, full);
    return 5.5 + 4 * (std::max(1.0, full) - 1) + pages * page < slack * ((p.d > 128 ? 14.3 : 10.3) + 0.7 * units * pages * kib / 5500);
}
// The same by the rows that a window leaves.  A prefix may hold any rows beside them, how many is on the device: then only where all of a unit's would not take much longer, either.
bool alone_by_window(const nkv_pages &p, const PromptArgs &a, int n_q_heads, int n_new)
{
    if (a.window <= 0) return false;
    const int64_t pages = std::min<int64_t>(p.max_pages, ((int64_t)a.window + n_new) / NKV_PAGE_ROWS + 2);
    return alone(p, n_q_heads, n_new, pages) && (!a.prefix || alone(p, n_q_heads, n_new, p.max_pages, 1.5));
}

Cap cap_of(double cap, double scale)
{
    const double x = scale / cap;
    Cap c{};
    c.cap_log2 = pages_scale(cap), c.over_cap = (float)x;
    c.small = cap <= 64;
    // the coefficients' powers, and those of the products that they meet, stay well within fp32; otherwise no product is near
    c.near = -1.f;
    if (x >= 0x1p-14 && x <= 0x1p4 && cap >= 0x1p-8 && cap <= 0x1p16) {
        c.near = (float)(kNearBound / x);
        for (int i = 0; i < 4; ++i) c.near_by[i] = (float)(kNear[i] * cap * 1.4426950408889634 * pow(x, 2 * i + 1));
    }
    c.mid = c.near;                                                        // without a longer polynomial a column's logits are near or beyond, whatever its neighbours' are
    if (x >= 0x1p-10 && x <= 0x1p4 && cap >= 0x1p-4 && cap <= 0x1p16) {
        c.mid = (float)(kMidBound / x);
        for (int i = 0; i < 6; ++i) c.mid_by[i] = (float)(kMid[i] * cap * 1.4426950408889634 * pow(x, 2 * i + 1));
    }
    return c;
}

}  // namespace

bool pages_prompt_one_launch(const nkv_pages &p, int n_q_heads, int n_new)
{
    // fewer than 2^32 threads: 512 a workgroup of the products, and a thread for four dims of a column where parts are joined
    const int64_t units = (int64_t)p.n_seqs * p.H, cols = (int64_t)(n_q_heads / p.H) * n_new;
    return cols < (1 << 30) && units * ((cols + 127) / 128) < (1 << 23) && (!few_columns(p, n_q_heads, n_new) || units * cols < (1 << 24));
}

size_t pages_prompt_ws_bytes(const nkv_pages &p, int n_q_heads, int n_new)
{
    if (alone(p, n_q_heads, n_new, p.max_pages)) return 0;
    if (few_columns(p, n_q_heads, n_new)) return prompt_token_ws_bytes(p, n_q_heads, n_new);
    const Grid g = grid_of(p, n_q_heads, n_new);
    return g.splits == 1 ? 0 : (size_t)g.splits * p.n_seqs * (n_q_heads * (size_t)n_new) * (p.d + 4) * sizeof(float);
}

hipError_t launch_pages_prompt(const void *q, const nkv_pages &p, const nkv_logit_rules *rules, int n_q_heads, int n_new, double scale, void *out, float *lse,
                               void *ws, hipStream_t st)
{
    PromptArgs a{};
    a.q = (const uint16_t *)q, a.pool = (const uint8_t *)p.pool, a.table = p.table, a.lens = p.lens;
    a.n_units = p.n_seqs * p.H, a.H = p.H, a.G = n_q_heads / p.H, a.n_new = n_new, a.n_pages = p.n_pages, a.max_pages = p.max_pages;
    a.scale_log2 = pages_scale(scale);
    a.flat = a.scale_log2 == 0.f;
    if (a.flat) a.scale_log2 = 1.f;
    a.flip = scale < 0 ? 0x80008000u : 0u;
    if (rules) {
        a.window = rules->window, a.slopes = rules->slopes, a.prefix = rules->prefix;
        if (rules->cap > 0) a.cap = cap_of(rules->cap, a.flat ? rules->cap : fabs(scale));
        a.bent = rules->cap > 0 || rules->slopes;
    }
    a.out = (uint16_t *)out, a.lse = lse, a.part = (float *)ws;
    if (alone(p, n_q_heads, n_new, p.max_pages) || alone_by_window(p, a, n_q_heads, n_new)) return launch_prompt_units(a, p, st);
    if (few_columns(p, n_q_heads, n_new)) return launch_prompt_tokens(a, p, ws, st);
    const Grid g = grid_of(p, n_q_heads, n_new);
    a.tiles = g.tiles, a.splits = g.splits;
    switch (p.d) {
    case 64: return launch_prompt_tiles<64>(a, p, st);
    case 96: return launch_prompt_tiles<96>(a, p, st);
    case 128: return launch_prompt_tiles<128>(a, p, st);
    case 192: return launch_prompt_tiles<192>(a, p, st);
    default: return launch_prompt_tiles<256>(a, p, st);
    }
}

}  // namespace nkv
