// Attention of many columns over pages, with rules for the logits (nkv_pages_prompt_attention): what is shared by its two kernels, and that of a prompt's
// chunk.  A column is a token and a query head of a KV head: column t G + g of a unit.
#pragma once

#include "nkv_pages.h"

namespace nkv {

// What a call asks for, on its way to the kernels.
struct PromptArgs {
    const uint16_t *q;
    const uint8_t *pool;
    const int32_t *table, *lens;
    int32_t n_units, H, G, n_new, n_pages, max_pages;
    float scale_log2;                    // positive, subnormal or not
    uint32_t flip;                       // sign bits of the query that change: those of a negative scale
    bool flat;                           // a scale of zero: the query counts as zeros
    bool bent;                           // cap or slopes
    float cap_log2, over_cap;            // cap * log2(e) and scale / cap; 0: no cap
    int32_t window;                      // 0: none
    const float *slopes;                 // [H * G]
    const int32_t *prefix;               // [sequences]
    uint16_t *out;
    float *lse, *part;                   // part: [split][unit][column][D + 4]: weighted values, maximum, sum
    int32_t tiles, splits;
};

constexpr float kNoMax = -3.0e38f;       // running maximum before any row was seen
constexpr float kFarMax = 0x1p24f;       // from here on a maximum's last place is 2 or more: logits are rounded as it is before they are taken from it
constexpr float kToLn = 0.6931471805599453f, kToLog2 = 1.4426950408889634f;

// The rows that the tokens on rows r0 .. r1 of a unit see, in pages: `front` from the first page on, then those from page front + skip on.
struct Seen {
    int front, skip, count;
    __device__ __forceinline__ int page(int step) const { return step < front ? step : step + skip; }
};
__device__ __forceinline__ Seen seen_pages(int r0, int r1, int window, int prefix)
{
    if (r1 < 0) return {0, 0, 0};
    const int lo = window > 0 ? max(0, r0 - window + 1) / kRows : 0, all = (prefix + kRows - 1) / kRows, front = min(all, lo);
    return {front, lo - front, front + max(r1 / kRows + 1, all) - lo};
}
__device__ __forceinline__ int rows_of(int len, int max_pages) { return max(0, min(len, max_pages * kRows)); }

// A logit in powers of two from a product: capped, less its distance's share.  |x| <= 5/8: x (1 - 0.33 x^2 + ..), a minimax polynomial whose relative error is 2^-27.9;
// beyond: (1 - e^-2x) / (1 + e^-2x), where nothing cancels.
template <int N> __device__ __forceinline__ void bend(float (&s)[N], float scale_log2, float cap_log2, float over_cap)
{
    if (cap_log2 == 0.f) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] *= scale_log2;
        return;
    }
    float far = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] *= over_cap;
        far = fmaxf(far, fabsf(s[i]));
    }
    const bool any_far = __any(far > 0.625f);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float x = s[i], y = x * x;
        float p = fmaf(y, -0.005659991875290871f, 0.020591000095009804f);
        p = fmaf(y, p, -0.053721074014902115f);
        p = fmaf(y, p, 0.13331127166748047f);
        p = fmaf(y, p, -0.3333325982093811f);
        p = fmaf(y, p, 1.f) * x;
        if (any_far) {
            const float e = __builtin_amdgcn_exp2f(fabsf(x) * (-2.f * kToLog2));
            const float t = (1.f - e) * __builtin_amdgcn_rcpf(1.f + e);
            p = fabsf(x) > 0.625f ? copysignf(t, x) : x != x ? x : p;
        }
        s[i] = p * cap_log2;
    }
}

size_t prompt_token_ws_bytes(const nkv_pages &p, int n_q_heads, int n_new);
hipError_t launch_prompt_tokens(const PromptArgs &a, const nkv_pages &p, void *ws, hipStream_t st);

// Wavefronts of a workgroup, of 32 columns each: eight, or four where a lane's queries and weighted values take more than half of its registers.
constexpr int prompt_waves(int d, bool two_pieces) { return d > 128 || (d == 128 && two_pieces) ? 4 : 8; }
template <int D> hipError_t launch_prompt_tiles(const PromptArgs &a, const nkv_pages &p, hipStream_t st);

}  // namespace nkv
