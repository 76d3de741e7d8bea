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

#include "roles.h"

namespace retro {

inline bool is_mx4(const Geometry& g) { return (g.flags & RETRO_FLAG_KV_MX4) != 0; }

// launch_append_tokens, launch_prefill and launch_update_kv (mx4_store.hip); sources and
// cache 16-byte aligned.  `counters`: those of the score launch that selects behind the
// append in the same step, set to zero by it.
hipError_t launch_mx4_append_tokens(const Geometry& g, int step, const retro_kv_cache& c, int n_tok,
                                    const void* k_new, const void* v_new, hipStream_t s,
                                    int32_t* counters = nullptr);
hipError_t launch_mx4_prefill(const Geometry& g, const retro_kv_cache& c, int seq, int start, int n,
                              const void* k_src, const void* v_src, hipStream_t s);
hipError_t launch_mx4_update_kv(const Geometry& g, const retro_kv_cache& c, int n, const void* k_upd,
                                const void* v_upd, hipStream_t s);

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
typedef uint32_t mx4_u32x4 __attribute__((ext_vector_type(4)));
template <typename T>
__device__ __forceinline__ mx4_u32x4 mx4_piece(uint32_t codes, float scale) {
  if constexpr (sizeof(T) == 2) {
    return mx4_u32x4{mx4_bf16<0>(codes, scale), mx4_bf16<1>(codes, scale), mx4_bf16<2>(codes, scale),
                 mx4_bf16<3>(codes, scale)};
  } else {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
    const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
    return mx4_u32x4{__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1])};
  }
}

// A lane's piece of a head's vector in codes; the lanes of a block together.
template <typename T>
struct Codes {
  static constexpr int E = 16 / sizeof(T);
  uint32_t codes;  // E of them
  int e;
  __device__ explicit Codes(mx4_u32x4 piece) {
    float x[E];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        x[2 * i] = __uint_as_float(piece[i] << 16);
        x[2 * i + 1] = __uint_as_float(piece[i] & 0xffff0000u);
      } else {
        x[i] = __uint_as_float(piece[i]);
      }
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max(top, (uint32_t)dpp_i<kDppXor1>((int)top));
    top = max(top, (uint32_t)dpp_i<kDppXor2>((int)top));
    if constexpr (E == 4) top = max(top, (uint32_t)dpp_i<kDppHalfMirror>((int)top));
    e = mx4_exponent(top);
    // (a block that is NaN as a whole has codes like any other)
    const float s = mx4_scale(e == kMx4NaN ? 127 : e);
    codes = mx4_encode<0>(0, x[0], x[1], s);
    codes = mx4_encode<1>(codes, x[2], x[3], s);
    if constexpr (E == 8) {
      codes = mx4_encode<2>(codes, x[4], x[5], s);
      codes = mx4_encode<3>(codes, x[6], x[7], s);
    }
  }
  __device__ mx4_u32x4 values() const { return mx4_piece<T>(codes, mx4_scale(e)); }
  // The codes to their places: of token t of a page whose keys (values) are at `block`, the
  // lane being number c of a vector.
  template <int PS, int D>
  __device__ void store_key(char* block, int t, int c) const {
    put(block + t * (D / 2) + c * (E / 2));
    if (c * E % 32 == 0) block[PS * D / 2 + t * (D / 32) + c * E / 32] = (char)e;
  }
  template <int PS, int D>
  __device__ void store_value(char* block, int t, int c) const {
    char* group = block + t / 4 * (2 * D);
    const int part = c * E / (D / 16), in = c * E % (D / 16);
    if constexpr (E <= D / 16) {
      put(group + (part * 4 + t % 4) * (D / 32) + in / 2);
    } else {  // (two parts of four elements)
      static_assert(E == 2 * (D / 16), "a piece is a part, or half of one, or two");
      reinterpret_cast<uint16_t*>(group)[part * 4 + t % 4] = (uint16_t)codes;
      reinterpret_cast<uint16_t*>(group)[part * 4 + 4 + t % 4] = (uint16_t)(codes >> 16);
    }
    if (c * E % 32 == 0) block[PS * D / 2 + (t / 4 * (D / 32) + c * E / 32) * 4 + t % 4] = (char)e;
  }

 private:
  __device__ void put(char* at) const {
    if constexpr (E == 8) *reinterpret_cast<uint32_t*>(at) = codes;
    else *reinterpret_cast<uint16_t*>(at) = (uint16_t)codes;
  }
};

}  // namespace retro
