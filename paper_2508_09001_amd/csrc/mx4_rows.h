// What a wavefront does with 32 tokens of a cache in 4 bits and up to NR tiles of 16 rows
// (a row: a query of one head of the group), shared by the attention kernels.
//
// S^T = K Q^T and O^T += V^T P^T on 16 x 16 x 32 products, 16 tokens of each tile's
// scores to a product, with operands made in registers: a lane reads its codes (a quarter of a key;
// four tokens' elements of a sixteenth of the vector) straight from the page, and the converted
// values are the operand.  The order within a contraction is free as long as both operands have it:
// lane l's share of key l % 16 is the block l / 16 of the vector as it lies, and its queries the
// same elements; row i of product number p of the outputs is element (d / 16) i + p, so that one
// piece of a value page feeds all of them.  A lane ends up with the scores of tokens 4 (l / 16) ..
// + 3 of both halves of its row l % 16, which are the weights that it needs for the second product,
// so that nothing moves between lanes.
//
// fp32 rows are taken apart into three bf16 terms (8 bits each: all of the 24), queries
// and weights alike; the values of codes are exact in bf16, so that products are exact
// and sums in fp32, in three matrix instructions instead of the sixteen times slower
// ones of fp32.  Weights of bf16 rows are two terms or three (PT), each what the rounding
// of those before it leaves.
#pragma once

#include "mx4.h"
#include "roles.h"

namespace retro {
namespace {

// 32 tokens of a head as they lie in the page(s): half t is 16 of them.
template <int D>
struct Mx4Tile {
  static constexpr int W = D / 32;  // words of a lane's piece
  uint32_t k[2][W], v[2][W];
  uint32_t ke[2], ve[2];            // exponent of the key's piece, of the four values
};

// Where a lane's pieces of 16 tokens lie behind the first one's place in the page.
template <int D, int P>
struct Mx4Places {
  uint32_t k, v, ke, ve;  // (unsigned: added to a scalar address by the load itself)
  __device__ __forceinline__ explicit Mx4Places(int lane) {
    const int r = lane & 15, quarter = lane >> 4;
    k = r * (D / 2) + quarter * (D / 8);
    v = lane * (D / 8);
    ke = P * D / 2 + r * (D / 32) + quarter * (D / 32) / 4;
    ve = P * D / 2 + (quarter * (D / 32) + r * (D / 16) / 32) * 4;
  }
  // keys, or values, of half t of a tile: 16 tokens from `slot` on of the page at `block`.
  // ONCE: not kept in the caches.
  template <bool ONCE>
  __device__ __forceinline__ void load_keys(Mx4Tile<D>& x, int t, const char* block, int slot) const {
    piece<ONCE>(x.k[t], block + slot * (D / 2) + k);
    x.ke[t] = *reinterpret_cast<const uint8_t*>(block + slot * (D / 32) + ke);
  }
  template <bool ONCE>
  __device__ __forceinline__ void load_values(Mx4Tile<D>& x, int t, const char* block, int slot) const {
    piece<ONCE>(x.v[t], block + slot * (D / 2) + v);
    x.ve[t] = *reinterpret_cast<const uint32_t*>(block + slot * (D / 32) + ve);
  }
  template <bool ONCE>
  static __device__ __forceinline__ void piece(uint32_t (&to)[D / 32], const char* from) {
    typedef uint32_t words __attribute__((ext_vector_type(D / 32)));
    const words* p = reinterpret_cast<const words*>(from);
    words w;
    if constexpr (ONCE) w = __builtin_nontemporal_load(p);
    else w = *p;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) to[i] = w[i];
  }
};

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x05040100u);
}
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}
__device__ __forceinline__ uint32_t round_pair(float a, float b) {  // to bf16
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  uint32_t w = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
  asm("" : "+v"(w));  // one conversion for the pair: its halves are taken from w
  return w;
}
// what is left of x behind its upper 8 bits (nothing of an infinity)
__device__ __forceinline__ float below_bf16(float x) {
  const float top = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
  return fabsf(x) < INFINITY ? x - top : 0.f;
}

template <typename T, int D, int NR, int PT = sizeof(T) == 2 ? 2 : 3>
struct Mx4Rows {
  static constexpr int KK = D / 32;                      // products of a contraction over d
  static constexpr int DT = D / 16;                      // products of the outputs
  static constexpr int QT = sizeof(T) == 2 ? 1 : 3;      // terms of a query
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  bf16x8 q[NR][QT][KK];
  f32x4 acc[NR][DT];
  float m[NR], l[NR];  // running maximum of the scores (unscaled), the lane's sum
  float c;             // scale * log2(e)

  // row n's queries (the lane's row of it), zeros for one that does not exist
  __device__ __forceinline__ void start(int n, const T* row, bool live, int lane) {
    const T* mine = row + (lane >> 4) * (D / 4);
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < KK; ++i) {
        const u32x4 x = live ? reinterpret_cast<const u32x4*>(mine)[i] : u32x4{0, 0, 0, 0};
        q[n][0][i] = __builtin_bit_cast(bf16x8, x);
      }
    } else {
#pragma unroll
      for (int i = 0; i < KK; ++i) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const f32x4 y = live ? reinterpret_cast<const f32x4*>(mine)[2 * i + j] : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 4; ++e) x[4 * j + e] = y[e] != y[e] ? __builtin_nanf("") : y[e];  // NaN in its upper bits
        }
#pragma unroll
        for (int term = 0; term < 3; ++term) {
          u32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            w[e] = high_halves(__float_as_uint(x[2 * e]), __float_as_uint(x[2 * e + 1]));
          q[n][term][i] = __builtin_bit_cast(bf16x8, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = below_bf16(x[e]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[n] = -INFINITY;
    l[n] = 0.f;
  }

  // The tile's keys and values with the rows.  hide(n, s): -inf for scores that do not
  // count, s[t][e] that of the lane's row and token 16 t + 4 (lane / 16) + e.  keys_done, values_done:
  // the tile's keys, or values, are no longer needed.
  template <typename Hide, typename KeysDone, typename ValuesDone>
  __device__ __forceinline__ void step(const Mx4Tile<D>& x, Hide&& hide, KeysDone&& keys_done,
                                       ValuesDone&& values_done) {
    f32x4 s[NR][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int n = 0; n < NR; ++n) s[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
      const float scale = mx4_scale((int)x.ke[t]);
#pragma unroll
      for (int i = 0; i < KK; ++i) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = mx4_bf16(x.k[t][i], scale, e);
        const bf16x8 k = __builtin_bit_cast(bf16x8, w);
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int term = QT - 1; term >= 0; --term)
            s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[n][term][i], s[n][t], 0, 0, 0);
      }
    }
    keys_done();
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      hide(n, s[n]);
      float mx = s[n][0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[n][e / 4][e % 4]);
      // The maximum follows only when a weight would pass 2^8: weights of up to 256
      // lose nothing, and most steps leave the outputs as they are.
      if (wave_ballot((mx - m[n]) * c > 8.f)) {
        const float mn = fmaxf(m[n], col_max4(mx));
        const float alpha = __builtin_amdgcn_exp2f((m[n] - mn) * c);
        const float a = mn == -INFINITY ? 0.f : alpha;
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[n][i] *= a;
        l[n] *= a;
        m[n] = mn;
      }
    }
    bf16x8 p[NR][PT];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      // (the difference before the product: exact where scores are large)
      const float mu = m[n] == -INFINITY ? 0.f : m[n];
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = __builtin_amdgcn_exp2f((s[n][e / 4][e % 4] - mu) * c);
        l[n] += w[e];
      }
#pragma unroll
      for (int term = 0; term < PT; ++term) {
        u32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (sizeof(T) == 2) {
            y[e] = round_pair(w[2 * e], w[2 * e + 1]);
            w[2 * e] -= __uint_as_float(y[e] << 16);
            w[2 * e + 1] -= __uint_as_float(y[e] & 0xffff0000u);
          } else {
            y[e] = high_halves(__float_as_uint(w[2 * e]), __float_as_uint(w[2 * e + 1]));
            w[2 * e] -= __uint_as_float(__float_as_uint(w[2 * e]) & 0xffff0000u);
            w[2 * e + 1] -= __uint_as_float(__float_as_uint(w[2 * e + 1]) & 0xffff0000u);
          }
        }
        p[n][term] = __builtin_bit_cast(bf16x8, y);
      }
    }
    // (a scale's bits below its exponent field, and its sign, do not count)
    float vs[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      vs[t][0] = __uint_as_float(x.ve[t] << 23);
      vs[t][1] = __uint_as_float(x.ve[t] << 15);
      vs[t][2] = __uint_as_float(x.ve[t] << 7);
      vs[t][3] = __uint_as_float(x.ve[t] >> 1);
    }
#pragma unroll
    for (int j = 0; j < DT / 2; ++j) {
      u32x4 lo, hi;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = e * (DT / 2) + j;  // byte of the lane's piece: token e, elements 2 j, 2 j + 1
          w[e] = mx4_bf16(x.v[t][at / 4], vs[t][e], at % 4);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          lo[2 * t + e] = low_halves(w[2 * e], w[2 * e + 1]);
          hi[2 * t + e] = high_halves(w[2 * e], w[2 * e + 1]);
        }
      }
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int term = PT - 1; term >= 0; --term) {
          acc[n][2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), p[n][term],
                                                                  acc[n][2 * j], 0, 0, 0);
          acc[n][2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), p[n][term],
                                                                      acc[n][2 * j + 1], 0, 0, 0);
        }
    }
    values_done();
  }

  // A row's outputs that the lane holds: f(d, o) for pieces of four elements from d on.
  template <typename F>
  __device__ __forceinline__ void each(int n, int lane, F&& f) const {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < DT; i += 4)
        f(DT * (4 * (lane >> 4) + e) + i, f32x4{acc[n][i][e], acc[n][i + 1][e], acc[n][i + 2][e], acc[n][i + 3][e]});
  }
};

// Exponents of four values of which `live` (from the first one) hold a token: the others'
// are made finite ones, so that a weight of zero leaves nothing of their codes.
__device__ __forceinline__ uint32_t live_exponents(uint32_t ve, int live) {
  const uint32_t keep = live >= 4 ? ~0u : live <= 0 ? 0u : (1u << 8 * live) - 1;
  return (ve & keep) | (0x7f7f7f7fu & ~keep);
}

}  // namespace
}  // namespace retro
