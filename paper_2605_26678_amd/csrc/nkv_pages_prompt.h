// Attention of many columns over pages, with rules for the logits (nkv_pages_prompt_attention): what is shared by its two kernels, and that of a prompt's
// chunk.  A column is a token and a query head of a KV head: column t G + g of a unit.
#pragma once

#include "nkv_pages.h"

namespace nkv {

// A logit's cap: cap * log2(e) tanh(x), x = product * over_cap; none where cap_log2 is 0.  Products of up to `near` take near_by[0 .. 3] as the coefficients of
// product^1, 3, 5 and 7, those of up to `mid` (no less than near) take mid_by for those up to 11.
struct Cap {
    float cap_log2, over_cap, near, near_by[4], mid, mid_by[6];
    bool small;                          // up to 64
};

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
    Cap cap;
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
    const int lo = window > 0 ? max(0, max(r0, 0) - window + 1) / kRows : 0, all = (prefix + kRows - 1) / kRows, front = min(all, lo);
    return {front, lo - front, front + max(r1 / kRows + 1, all) - lo};
}
__device__ __forceinline__ int rows_of(int len, int max_pages) { return max(0, min(len, max_pages * kRows)); }

// A capped logit in powers of two from a product.  |x| <= 5/16, as most logits are that a cap is meant for: tanh(x) as x - x^3 / 3 + .., a minimax polynomial
// whose relative error is 2^-26, with the scale and the cap in its coefficients; |x| <= 5/8: a longer one, 2^-27.9; beyond: (1 - e^-2x) / (1 + e^-2x), which is off by 2^-23 at
// most, 64 * 2^-23 of a logit capped at 64.  Of larger caps' logits small ones keep to the polynomial, each by itself.  Every lane, which has one column, chooses by
// `most`, the largest of its products with rows that the column sees: no other rows have a part in how these are rounded.
constexpr double kNear[4] = {1.0, -0.33332862850586767, 0.13309054081886735, -0.049920588703130035}, kNearBound = 0.3125;
constexpr double kMid[6] = {1.0, -0.3333325982093811, 0.13331127166748047, -0.053721074014902115, 0.020591000095009804, -0.005659991875290871}, kMidBound = 0.625;
template <int N> __device__ __forceinline__ void bend(float (&s)[N], float most, const Cap &c)
{
    if (!__any(most > c.near)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = s[i] * s[i];
            s[i] *= fmaf(y, fmaf(y, fmaf(y, c.near_by[3], c.near_by[2]), c.near_by[1]), c.near_by[0]);
        }
        return;
    }
    const bool beyond = most > c.mid;
    float by[6];                                                           // (two zeros in front leave the short one's bits as they are)
#pragma unroll
    for (int k = 0; k < 6; ++k) by[k] = most > c.near ? c.mid_by[k] : k < 4 ? c.near_by[k] : 0.f;
    auto close = [&by](float x) {
        const float y = x * x;
        return x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, by[5], by[4]), by[3]), by[2]), by[1]), by[0]);
    };
    if (!__any(beyond)) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = close(s[i]);
        return;
    }
    auto far = [](float x) {
        const float e = __builtin_amdgcn_exp2f(fabsf(x) * (-2.f * kToLog2));
        return copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), x);
    };
    if (c.small) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = beyond ? far(s[i] * c.over_cap) * c.cap_log2 : close(s[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float x = s[i] * c.over_cap, y = x * x;
        float p = (float)kMid[5];
#pragma unroll
        for (int k = 4; k >= 0; --k) p = fmaf(y, p, (float)kMid[k]);
        s[i] = beyond ? (fabsf(x) > (float)kMidBound ? far(x) : p * x) * c.cap_log2 : close(s[i]);
    }
}

size_t prompt_token_ws_bytes(const nkv_pages &p, int n_q_heads, int n_new);
hipError_t launch_prompt_units(const PromptArgs &a, const nkv_pages &p, hipStream_t st);
hipError_t launch_prompt_tokens(const PromptArgs &a, const nkv_pages &p, void *ws, hipStream_t st);

// Wavefronts of a workgroup, of 32 columns each.  128 dims: eight, one workgroup a compute unit (a chunk of 2048 tokens and 32 heads behind 30720 rows 1120 us, with two of four
// 1230; 16 prompts of 512 tokens 87 and 94).  64 dims: four, three of them a compute unit (8 prompts of 509 tokens behind 300 that all see 26.9 us, with one of
// eight 34.6; that chunk 785 and 775).  96 dims: four, two of them (35 prompts of 547 tokens 112 and 127 us; that chunk 966 and 932).  More dims, and two pieces of 128: four, one of
// them, since a lane's queries and weighted values take more than half of its registers.
constexpr int prompt_waves(int d, bool two_pieces) { return d == 128 && !two_pieces ? 8 : 4; }
constexpr int prompt_groups(int d, bool two_pieces) { return d == 64 && !two_pieces ? 3 : d <= 96 ? 2 : 1; }   // workgroups a compute unit holds
template <int D> hipError_t launch_prompt_tiles(const PromptArgs &a, const nkv_pages &p, hipStream_t st);

}  // namespace nkv
