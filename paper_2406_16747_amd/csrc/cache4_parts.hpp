// The cache in 4 bits: what its append, its attention and its reading back share.
//
// A value is an e2m1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) times a power of two that 32 values share: of keys 32 channels of a token, of
// values 32 tokens of a channel.  The power is the smallest with which none of the 32 passes 6, so a value is off by a fifth of the
// largest at most (where that is 5 times the power, 4 stands for it), and scaling loses nothing.  Two exceptions: where the largest is above 6 * 2^125 the
// power stays 2^125 and 6 of them stand for it (off by a quarter of bf16's largest number, at most), and where it is below 2^-100 zeros do.  Inside a page codes and scales lie as the
// lanes of the matrix instructions take them, 16 bytes of codes to a lane at a time: the attention's loads are whole lines, straight into LDS.
#pragma once
#include "block_parts.hpp"

namespace spk {

constexpr int FORMAT_E2M1 = SPARSEK_E2M1;

// Bytes of a page: codes, and scales (biased by 127, 0: a group of zeros), of keys as of values.
template <int D>
struct Page4 {
    static constexpr int CODES = BT * D / 2, SCALES = BT * D / 32;
    // 8 codes (4 bytes): keys of token s, channels 8 c8 ..; values of channel c, tokens 8 s8 ..
    static __device__ __forceinline__ int key_at(int s, int c8)
    {
        const int t = s >> 2 & 3, row = (s >> 4) * 4 + (s & 3);
        if constexpr (D == 128) return ((t * 4 + c8 / 4) * 16 + row) * 16 + c8 % 4 * 4;
        else return ((t / 2 * 4 + c8 / 2) * 16 + row) * 16 + t % 2 * 8 + c8 % 2 * 4;
    }
    static __device__ __forceinline__ int value_at(int c, int s8) { return ((c / 32 * 4 + s8 / 2) * 16 + c % 16) * 16 + c / 16 % 2 * 8 + s8 % 2 * 4; }
    // the scale of token s, channels 32 j ..; of channel c, tokens 32 j ..
    static __device__ __forceinline__ int key_scale_at(int s, int j) { return (j * 16 + (s >> 4) * 4 + (s & 3)) * 4 + (s >> 2 & 3); }
    static __device__ __forceinline__ int value_scale_at(int c, int j) { return (j * 16 + c % 16) * (D / 16) + c / 16; }
};

// The scale of a group whose largest magnitude has the bits `top`: the smallest power of two with top <= 6 of them, at most 2^125 (6 2^126
// is no number any more), as its biased exponent.
__device__ __forceinline__ unsigned scale_of_top(unsigned top) { return top >= __float_as_uint(TINY_MAX) ? min((top + 0x3FFFFFu >> 23) - 2u, 252u) : 0u; }

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

// 8 bf16 values as codes; e: their scale.
__device__ __forceinline__ unsigned codes_e2m1(u32x4 x, unsigned e)
{
    const float scale = __uint_as_float(e << 23);
    const unsigned p[4] = {x[0], x[1], x[2], x[3]};   // (a bit cast of a vector's element takes the first one's bits)
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2v, p[0]), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2v, p[1]), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2v, p[2]), scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2v, p[3]), scale, 3);
    return e ? w : 0u;
}

// 8 codes times their scale, which bf16 holds exactly whatever it is; scale: its float's bits, 0 for a group of zeros.
__device__ __forceinline__ bf16x8 widen_e2m1(unsigned w, unsigned scale)
{
    const float f = __uint_as_float(scale);
    const bf16x2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 1);
    const bf16x2v c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// Byte x of four scales as such bits.
__device__ __forceinline__ unsigned scale_bits(unsigned scales, int x) { return (scales >> 8 * x & 255) << 23; }

// What ks and vs hold: a page's largest scale, times 1.5 where one that is not 0 is less than 2^-36 of it (a reader that widens to fp16 cannot hold both),
// NaN where a value is not finite, which is what the attention and reading back look for.
constexpr int WIDE = 36;
__device__ __forceinline__ float page_scale(float top, int lowest)
{
    if (!(top < INFINITY)) return __uint_as_float(0x7FC00000u);
    const int e = (int)scale_of_top(__float_as_uint(top));
    return __uint_as_float((unsigned)e << 23 | (lowest < e - WIDE ? 0x400000u : 0u));
}

}  // namespace spk
