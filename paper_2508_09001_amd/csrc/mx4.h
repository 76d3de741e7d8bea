// The paged cache in 4 bits (RETRO_FLAG_KV_MX4): blocks of 32 elements of a head's
// vector with one exponent byte e each, an element being the value of its code (a sign,
// two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6) times 2^(e - 127),
// the elements and scales of the OCP Microscaling Formats specification's MXFP4.
//
// The matrix cores' neighbours convert both ways: v_cvt_scalef32_pk_fp4_f32 rounds two
// floats over the scale to the nearest codes (ties to even, at most 6) and
// v_cvt_scalef32_pk_bf16_fp4 (and _f32_) gives two codes' values times the scale, of which
// it looks at the exponent field only.  Values are exact in bf16, so that products with
// them lose nothing that those of a bf16 cache do not.
//
// A page of a KV head, keys or values: P d / 2 bytes of codes, then P d / 32 exponents.
//   keys    codes [P][d], exponents [P][d / 32]: the lanes of a 16 x 16 x 32 product's
//           operand, key lane % 16, each read a quarter of a key, which is one block
//   values  codes [P / 4][16][4][d / 16], exponents [P / 4][d / 32][4]: lane l of the
//           product with the weights reads four tokens' elements (d / 16) (l % 16) .. of
//           them, tokens 4 (l / 16) .., as one piece, and four exponents as one word
#pragma once

#include "internal.h"

namespace retro {

inline bool is_mx4(const Geometry& g) { return (g.flags & RETRO_FLAG_KV_MX4) != 0; }

// Attention of the window over the selected pages (mx4_window.hip): launch_attend's
// arguments and partials, with the split of mx4_window_geometry(g), which the combine of
// the partials takes too; or, with o_out and l_out (a single split), launch_combine_merge's
// results of mode 0.
Geometry mx4_window_geometry(const Geometry& g);
hipError_t launch_mx4_window(const Geometry& g, int step, const void* q_window, const retro_kv_cache& c,
                             const retro_selection& sel, float* o_ws, float* l_ws, float* o_out, float* l_out,
                             hipStream_t s);

constexpr int mx4_block_bytes(int P, int D) { return P * D / 2 + P * D / 32; }

// Exponents lie between that of the smallest scale whose codes are normal in bf16 (the
// matrix cores need not keep others) and that of the largest whose codes are finite.
constexpr int kMx4Least = 2, kMx4Most = 252;
constexpr int kMx4NaN = 255;  // of a block with a NaN or an infinity: NaN throughout

// The exponent byte of a block whose largest magnitude has these bits: the scale that
// puts it at 4 .. 7 times, or 3.5 .. 4 instead of 7 .. 8, whose codes would be 6.  (Of
// normal values the root mean square error is 0.112; 0.115 with 7 .. 8 kept, 0.115 too
// where everything from 6 on takes the larger scale.)
__device__ __forceinline__ int mx4_exponent(uint32_t largest) {
  const int e = (int)((largest + (1u << 21)) >> 23) - 2;
  return largest >= 0x7f800000u ? kMx4NaN : min(max(e, kMx4Least), kMx4Most);
}
__device__ __forceinline__ float mx4_scale(int e) { return __uint_as_float((uint32_t)e << 23); }

// Codes of two values, byte SEL of the result (the others as in `old`).
template <int SEL>
__device__ __forceinline__ uint32_t mx4_encode(uint32_t old, float a, float b, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, scale, SEL);
}
// The values of byte SEL's two codes, as two bf16 (the low half's code low).
template <int SEL>
__device__ __forceinline__ uint32_t mx4_bf16(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}
__device__ __forceinline__ uint32_t mx4_bf16(uint32_t codes, float scale, int sel) {
  switch (sel) {  // (a constant after unrolling)
    case 0: return mx4_bf16<0>(codes, scale);
    case 1: return mx4_bf16<1>(codes, scale);
    case 2: return mx4_bf16<2>(codes, scale);
    default: return mx4_bf16<3>(codes, scale);
  }
}

// The values of the 16 / sizeof(T) codes at the low end of a word, as 16 bytes of T.
template <typename T>
__device__ __forceinline__ auto mx4_piece(uint32_t codes, float scale) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  if constexpr (sizeof(T) == 2) {
    return u32x4{mx4_bf16<0>(codes, scale), mx4_bf16<1>(codes, scale), mx4_bf16<2>(codes, scale),
                 mx4_bf16<3>(codes, scale)};
  } else {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
    const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
    return u32x4{__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1])};
  }
}

}  // namespace retro
