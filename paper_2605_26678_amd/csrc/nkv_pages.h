// Layout of a page of the paged cache and the 4-bit format's conversions, shared by the kernels that write and read pages.
#pragma once

#include "nkv_device.h"

#include <type_traits>

namespace nkv {

using u32x4 = unsigned int __attribute__((ext_vector_type(4)));
using u32x2 = unsigned int __attribute__((ext_vector_type(2)));
using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
using f16x2 = _Float16 __attribute__((ext_vector_type(2)));

constexpr int kRows = NKV_PAGE_ROWS;
constexpr int kBlock = 32;                       // dims that share a scale
// dims of a row that one lane of the product with V takes
constexpr int chunk_of(int D) { return D <= 64 ? 4 : D <= 128 ? 8 : 16; }

template <int D> struct Fp4Page {                // byte offsets inside a page
    static constexpr int C = chunk_of(D), NB = D / kBlock;
    static constexpr int kV = kRows * D / 2, kKScale = kRows * D, kVScale = kKScale + kRows * NB, kBytes = kVScale + kRows * NB;
    __device__ static int k_code(int row, int dim) { return row * (D / 2) + dim / 2; }
    __device__ static int v_code(int row, int dim) { return kV + ((row / 4 * (D / C) + dim / C) * 4 + row % 4) * (C / 2) + dim % C / 2; }
    __device__ static int k_scale(int row, int block) { return kKScale + (block * 16 + row % 16) * 4 + row / 16; }
    __device__ static int v_scale(int row, int block) { return kVScale + ((row / 4 % 4 * NB + block) * 4 + row / 16) * 4 + row % 4; }
};
template <int D> struct WidePage {               // 16-bit rows
    static constexpr int kV = kRows * D * 2, kBytes = 2 * kV;
    __device__ static int k(int row, int dim) { return (row * D + dim) * 2; }
    __device__ static int v(int row, int dim) { return kV + (row * D + dim) * 2; }
};

template <bool F16> __device__ __forceinline__ void unpack8(const u32x4 &r, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = r[i];
        if constexpr (F16) {
            const f16x2 h = __builtin_bit_cast(f16x2, w);
            x[2 * i] = (float)h.x;
            x[2 * i + 1] = (float)h.y;
        } else {
            x[2 * i] = __uint_as_float(w << 16);
            x[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
        }
    }
}
template <bool F16> __device__ __forceinline__ u32x4 pack8(const float (&x)[8])      // to nearest, ties to even
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (F16) r[i] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)x[2 * i], (_Float16)x[2 * i + 1]});
        else r[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
    }
    return r;
}

// Scale byte of the block that four neighbouring lanes hold eight values each of: with the largest magnitude in [1, 2) * 2^e the
// scale is 2^(e - 2), and twice that from 1.75 * 2^e on, where the largest code, 6, would be off by more than a rounding.  Compared as
// integers, so that a NaN counts as the largest.  All four lanes are active.
__device__ __forceinline__ uint32_t fp4_scale(const float (&x)[8])
{
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max(top, dpp_word<0xB1>(top));         // quad_perm [1,0,3,2]
    top = max(top, dpp_word<0x4E>(top));         // quad_perm [2,3,0,1]
    const uint32_t e = top >> 23;
    if (e == 255u) return 255u;
    const int s = (int)e - 2 + ((top & 0x600000u) == 0x600000u ? 1 : 0);
    return (uint32_t)max(s, 1);
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight codes of a block with that scale, dim i at bits 4 i.  (The instruction divides by the scale and rounds to nearest, ties to even.)
__device__ __forceinline__ uint32_t fp4_codes(const float (&x)[8], uint32_t scale)
{
    const float s = scale_value(scale);
    uint32_t w = 0u;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
    return scale == 255u ? 0u : w;
}
// Eight values in the rows' type, those beyond its largest finite one as that, NaN for scale 255.
template <bool F16> __device__ __forceinline__ u32x4 fp4_rows(uint32_t w, uint32_t scale)
{
    const float s = scale_value(scale);
    u32x4 r;
    if constexpr (F16) {
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 0)), r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 1));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 2)), r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 3));
    } else {
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0)), r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2)), r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
    }
    if (scale >= (F16 ? 141u : 253u)) {                                    // seldom: 6 * 2^14 and 6 * 2^126 are beyond the types
        constexpr uint32_t most = F16 ? 0x7bffu : 0x7f7fu;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t code = w >> (4 * i) & 15u, sign = (code & 8u) << 12;
            // magnitudes but 0 as 2^e * 1 or 1.5: the codes 1, 2 .. 7 are 2^-1, 2^0 .. 1.5 * 2^2 times the scale
            const int e = (int)scale - 127 + (int)((code & 7u) >> 1) - 1;
            const bool beyond = (code & 7u) != 0u && e > (F16 ? 15 : 127);
            const uint32_t h = scale == 255u ? 0x7fffu : sign | most;
            if (scale == 255u || beyond) r[i / 2] = i % 2 ? (r[i / 2] & 0xffffu) | h << 16 : (r[i / 2] & 0xffff0000u) | h;
        }
    }
    return r;
}

// The eight codes of dims 8 c .. 8 c + 7 of V row `row`, which lie in one piece (or two, of head dims up to 64).
template <int D> __device__ __forceinline__ void store_v_codes(uint8_t *page, int row, int c, uint32_t w)
{
    using P = Fp4Page<D>;
    uint8_t *at = page + P::v_code(row, 8 * c);
    if constexpr (P::C == 4) {
        *reinterpret_cast<uint16_t *>(at) = (uint16_t)w;
        *reinterpret_cast<uint16_t *>(page + P::v_code(row, 8 * c + 4)) = (uint16_t)(w >> 16);
    } else {
        *reinterpret_cast<uint32_t *>(at) = w;
    }
}
template <int D> __device__ __forceinline__ uint32_t load_v_codes(const uint8_t *page, int row, int c)
{
    using P = Fp4Page<D>;
    const uint8_t *at = page + P::v_code(row, 8 * c);
    if constexpr (P::C == 4)
        return *reinterpret_cast<const uint16_t *>(at) | (uint32_t) * reinterpret_cast<const uint16_t *>(page + P::v_code(row, 8 * c + 4)) << 16;
    else return *reinterpret_cast<const uint32_t *>(at);
}

// f(std::integral_constant<int, D>) for the head dims that pages have.
template <typename F> inline bool for_head_dim(int d, F f)
{
    switch (d) {
    case 64: f(std::integral_constant<int, 64>{}); return true;
    case 96: f(std::integral_constant<int, 96>{}); return true;
    case 128: f(std::integral_constant<int, 128>{}); return true;
    case 192: f(std::integral_constant<int, 192>{}); return true;
    case 256: f(std::integral_constant<int, 256>{}); return true;
    default: return false;
    }
}

}  // namespace nkv
