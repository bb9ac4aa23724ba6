// nkv_pages_prompt_attention for a token or a few: bound by memory, so with the kernels of nkv_pages_attention.
#include "nkv_pages_columns.h"

namespace nkv {

size_t prompt_token_ws_bytes(const nkv_pages &p, int n_q_heads, int n_new) { return columns_ws_bytes(p, n_q_heads, n_new); }

namespace {

AttendArgs args_of(const PromptArgs &c)
{
    AttendArgs a{};
    a.q = c.q, a.pool = c.pool, a.table = c.table, a.lens = c.lens;
    a.n_units = c.n_units, a.H = c.H, a.G = c.G, a.n_new = c.n_new, a.n_pages = c.n_pages, a.max_pages = c.max_pages;
    a.scale_log2 = c.scale_log2, a.flip = c.flip, a.flat = c.flat;
    a.bent = c.bent, a.cap = c.cap, a.window = c.window, a.slopes = c.slopes, a.prefix = c.prefix;
    a.out = c.out, a.lse = c.lse;
    return a;
}

}  // namespace

hipError_t launch_prompt_units(const PromptArgs &c, const nkv_pages &p, hipStream_t st) { return launch_units(args_of(c), p, st); }

hipError_t launch_prompt_tokens(const PromptArgs &c, const nkv_pages &p, void *ws, hipStream_t st)
{
    const AttendArgs a = args_of(c);
    if (p.dtype == NKV_DTYPE_F16) return launch_columns<true>(a, p, (_Float16 *)c.out, c.lse, ws, st);
    return launch_columns<true>(a, p, (__bf16 *)c.out, c.lse, ws, st);
}

}  // namespace nkv
