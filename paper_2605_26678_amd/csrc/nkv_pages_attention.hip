// Attention of a sequence's last tokens over its pages (nkv_pages_attention).
#include "nkv_pages_columns.h"

namespace nkv {

size_t pages_ws_bytes(const nkv_pages &p, int n_q_heads, int n_new) { return columns_ws_bytes(p, n_q_heads, n_new); }

hipError_t launch_pages_attention(const void *q, const nkv_pages &p, int n_q_heads, int n_new, double scale, float *out, float *lse, void *ws,
                                  hipStream_t st)
{
    AttendArgs a{};
    a.q = (const uint16_t *)q, a.pool = (const uint8_t *)p.pool, a.table = p.table, a.lens = p.lens;
    a.n_units = p.n_seqs * p.H, a.H = p.H, a.G = n_q_heads / p.H, a.n_new = n_new, a.n_pages = p.n_pages, a.max_pages = p.max_pages;
    a.scale_log2 = pages_scale(scale);
    a.flat = a.scale_log2 == 0.f;
    if (a.flat) a.scale_log2 = 1.f;
    a.flip = scale < 0 ? 0x80008000u : 0u;
    return launch_columns<false>(a, p, out, lse, ws, st);
}

}  // namespace nkv
