// nkv_pages_prompt_attention: which kernel takes a call.
#include "nkv_pages_prompt.h"

#include <algorithm>

namespace nkv {
namespace {

// Tables of up to that many pages: all rows in one launch.  (8 KV heads of 400 rows: 14 us so, shared out 12; of 64 rows 7.5, single tokens' kernels 11.5)
constexpr int kShort = 4;

struct Grid {
    int tiles, splits;                   // workgroups of a unit: tiles of columns, and shares of the rows that one sees
};
// Where the tiles are few, the rows are shared out too, until there is a workgroup for (nearly) every compute unit.  (More than one of them, where it holds more, would have twice the
// parts to write and join.)
Grid grid_of(const nkv_pages &p, int n_q_heads, int n_new)
{
    const int64_t cols = (int64_t)(n_q_heads / p.H) * n_new, at_once = 32 * prompt_waves(p.d, p.dtype == NKV_DTYPE_F16 && p.format == NKV_PAGES_FP4);
    const int64_t tiles = (cols + at_once - 1) / at_once, groups = (int64_t)p.n_seqs * p.H * tiles;
    return {(int)tiles, p.max_pages <= kShort ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(256 / groups, p.max_pages / 2))};
}

// Whether a call goes with the single tokens' kernels.  They share out all units' pages evenly and take up to 16 columns at a time, in some 10 us and what memory takes; the
// tiles take a page a microsecond in each workgroup whatever the columns, in one launch or two.  us, theirs / tiles, 8 KV heads of 128 dims:
//   4 bits    16 columns: 1024 rows of 1, 32 sequences 10.6 / 11.6, 22 / 29; 16384 rows 15 / 24, 110 / 364
//             32 columns: 1024 rows 11.1 / 11.8, 40 / 29; 4096 rows 12 / 16, 73 / 95; 16384 rows 24 / 25, 214 / 365
//             64 columns: 4096 rows 15 / 19, 140 / 97;  one column, 3 rows of 33 sequences with 32 heads 15 / 29
//   16 bits   8 columns: 600 rows 11.8 / 10.1, 25 / 19; 1024 rows 12.5 / 10.9, 39 / 28; 4096 rows 12.5 / 13.6, 92 / 96; 16384 rows 21 / 23, 284 / 354
//             32 columns: 4096 rows 19 / 16, 208 / 98
bool few_columns(const nkv_pages &p, int n_q_heads, int n_new)
{
    const int64_t cols = (int64_t)(n_q_heads / p.H) * n_new;
    if (p.max_pages <= kShort && p.n_seqs * p.H <= 512) return false;
    return p.format == NKV_PAGES_FP4 ? cols <= (p.max_pages > 32 ? 32 : 16) : cols <= 16 && p.max_pages > 20;
}

Cap cap_of(double cap, double scale)
{
    const double x = scale / cap;
    Cap c{};
    c.cap_log2 = pages_scale(cap), c.over_cap = (float)x;
    c.small = cap <= 64;
    // the coefficients' powers, and those of the products that they meet, stay well within fp32; otherwise no product is near
    c.near = c.mid = -1.f;
    if (x >= 0x1p-14 && x <= 0x1p4 && cap >= 0x1p-8 && cap <= 0x1p16) {
        c.near = (float)(kNearBound / x);
        for (int i = 0; i < 4; ++i) c.near_by[i] = (float)(kNear[i] * cap * 1.4426950408889634 * pow(x, 2 * i + 1));
    }
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
