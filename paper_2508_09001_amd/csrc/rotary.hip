// Per-head norms with the rotation by position: on queries and keys by
// themselves, and on the way into the paged cache.
//
// A head's vector is read as 16-byte pieces by LPV = d / E consecutive lanes.
// Its mean square is a sum over these lanes; a rotated pair lies in one lane
// (interleaved) or in two lanes rot_dim / 2 elements apart, which exchange their
// pieces as read (four words instead of eight products).  Norm, rotation and
// everything between stay in fp32 and are rounded once.  Bound by HBM: every
// vector is read once and written once, at 4.6 to 4.7 TB/s where a plain copy
// reaches 4.8; by the launch for a few rows.
#include "roles.h"
#include "rotary.h"

namespace retro {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__global__ void __launch_bounds__(256) rotary_table_kernel(float* __restrict__ table, int64_t n,
                                                           int half, int rot, double log2_base) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t p = i / half;
    const int e = (int)(i - p * half);
    double s, c;
    sincos((double)p * exp2(-2.0 * e / rot * log2_base), &s, &c);
    table[2 * i] = (float)c;
    table[2 * i + 1] = (float)s;
  }
}

template <typename T>
__device__ __forceinline__ void unpack(u32x4 w, float* x) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
  }
}

template <typename T>
__device__ __forceinline__ u32x4 pack(const float* y) {
  u32x4 w;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      w[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)y[2 * i], (__bf16)y[2 * i + 1]});
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(y[i]);
  }
  return w;
}

// What lane `c` of a vector's LPV lanes needs besides its piece.
template <typename T, int D>
struct Turn {
  static constexpr int E = 16 / sizeof(T);
  static constexpr int LPV = D / E;
  int c, rot, half, positions, interleaved;
  float eps;
  const float* table;

  __device__ Turn(const retro_rotary& r, int lane)
      : c(lane % LPV), rot(r.rot_dim), half(r.rot_dim / 2), positions(r.positions),
        interleaved(r.interleaved), eps(r.eps), table(r.table) {}

  // the lane that holds the other halves of this one's pairs
  __device__ int partner(int lane) const {
    const int i0 = c * E;
    if (interleaved || i0 >= rot) return lane;
    return i0 < half ? lane + half / E : lane - half / E;
  }

  // cosines and sines of the piece's pairs, (c, s) each; zero angle where nothing turns
  struct Angles {
    float cs[2 * E];
  };
  __device__ void angles(int pos, Angles& a) const {
    const int i0 = c * E;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      a.cs[2 * i] = 1.f;
      a.cs[2 * i + 1] = 0.f;
    }
    if (i0 >= rot) return;
    if (pos >= positions) {
#pragma unroll
      for (int i = 0; i < 2 * E; ++i) a.cs[i] = __builtin_nanf("");
      return;
    }
    const float* t = table + (int64_t)pos * rot;
    if (interleaved) {
#pragma unroll
      for (int i = 0; i < E; i += 4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(t + i0 + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) a.cs[i + e] = v[e];
      }
    } else {
      const int j = i0 < half ? i0 : i0 - half;
#pragma unroll
      for (int i = 0; i < 2 * E; i += 4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(t + 2 * j + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) a.cs[i + e] = v[e];
      }
    }
  }

  // the weights of a norm for the lane's piece and its partner's, as stored
  struct Weights {
    u32x4 own, other;
  };
  __device__ void weights(const void* w, Weights& out) const {
    out.own = out.other = u32x4{0, 0, 0, 0};
    if (!w) return;
    out.own = reinterpret_cast<const u32x4*>(w)[c];
    out.other = reinterpret_cast<const u32x4*>(w)[partner(c)];
  }

  __device__ u32x4 operator()(u32x4 raw, bool norm, const Weights& w, const Angles& a,
                              int lane) const {
    float x[E], y[E], z[E];
    unpack<T>(raw, x);
    const int p = partner(lane);
    u32x4 other;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      other[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(p * 4, (int)raw[i]);
    unpack<T>(other, z);
    if (norm) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
      ss += dpp_f<kDppXor1>(ss);
      ss += dpp_f<kDppXor2>(ss);
      ss += dpp_f<kDppHalfMirror>(ss);
      if constexpr (LPV >= 16) ss += dpp_f<kDppMirror>(ss);
      if constexpr (LPV >= 32) ss = rows_pair_sum(ss);
      const float r = 1.0f / sqrtf(ss * (1.0f / D) + eps);
      float own[E], theirs[E];
      unpack<T>(w.own, own);
      unpack<T>(w.other, theirs);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        x[i] = x[i] * r * own[i];
        z[i] = z[i] * r * theirs[i];
      }
    }
    if (interleaved) {
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        const float co = c * E < rot ? a.cs[i] : 1.f, si = c * E < rot ? a.cs[i + 1] : 0.f;
        y[i] = x[i] * co - x[i + 1] * si;
        y[i + 1] = x[i + 1] * co + x[i] * si;
      }
    } else {
      const float sign = c * E < half ? -1.f : 1.f;
#pragma unroll
      for (int i = 0; i < E; ++i) y[i] = x[i] * a.cs[2 * i] + sign * (z[i] * a.cs[2 * i + 1]);
    }
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (c * E >= rot) y[i] = x[i];
    return pack<T>(y);
  }
};

// One wavefront per row and ITER times 64 / LPV heads (queries' first, then keys'):
// the row's angles are read once for them, and their pieces are on the way together.
template <typename T, int D, int ITER>
__global__ void __launch_bounds__(256) rotate_qk_kernel(
    retro_rotary r, const int32_t* __restrict__ positions, int rows, int heads_q, int heads_k,
    const T* q, int64_t q_stride, const T* k, int64_t k_stride, T* q_out, T* k_out) {
  using Tn = Turn<T, D>;
  constexpr int VPW = 64 / Tn::LPV;
  const int lane = threadIdx.x & 63;
  const int heads = heads_q + heads_k, groups = (heads + ITER * VPW - 1) / (ITER * VPW);
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int row = (int)(unit / groups);
  const int head0 = (int)(unit - (int64_t)row * groups) * ITER * VPW + lane / Tn::LPV;
  if (row >= rows || head0 >= heads) return;
  const int pos = positions ? positions[row] : 0;
  const Tn turn(r, lane);
  u32x4 raw[ITER];
  typename Tn::Weights wq, wk;
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    const int head = min(head0 + i * VPW, heads - 1);
    const T* src = head < heads_q ? q + row * q_stride + head * D
                                  : k + row * k_stride + (head - heads_q) * D;
    raw[i] = reinterpret_cast<const u32x4*>(src)[turn.c];
  }
  if (pos < 0) return;
  turn.weights(r.q_norm, wq);
  turn.weights(r.k_norm, wk);
  typename Tn::Angles a;
  turn.angles(pos, a);
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    const int head = head0 + i * VPW;
    if (head >= heads) return;
    const bool is_q = head < heads_q;
    T* dst = is_q ? q_out + ((int64_t)row * heads_q + head) * D
                  : k_out + ((int64_t)row * heads_k + head - heads_q) * D;
    const u32x4 y = turn(raw[i], (is_q ? r.q_norm : r.k_norm) != nullptr, is_q ? wq : wk, a, lane);
    u32x4* at = reinterpret_cast<u32x4*>(dst) + turn.c;
    if (ITER > 1) __builtin_nontemporal_store(y, at);  // more than the L2s hold
    else *at = y;
  }
}

// ---- append ------------------------------------------------------------------------

// pages that a run touches
__device__ __forceinline__ int run_pages(const Run& r, int P) {
  if (r.n <= 0) return 0;
  return (int)(((int64_t)r.pos + r.n - 1) / P) - r.pos / P + 1;
}

// The sequence that unit `u` of all sequences' pages belongs to, and the page
// within its run; -1 behind the last.  Every wavefront finds it by itself.
__device__ __forceinline__ int find_page(const retro_chunk& ch, int batch, int P, int lane, int u,
                                         Run& run, int& page) {
  int base = 0;
  for (int b0 = 0; b0 < batch; b0 += 64) {
    Run r{0, 0, 0};
    if (b0 + lane < batch) r = chunk_run(ch, b0 + lane);
    const int n = run_pages(r, P), upto = base + wave_inclusive_scan(n);
    const uint64_t past = wave_ballot(upto > u);
    if (past) {
      const int l = __builtin_ctzll(past);
      run.row = __builtin_amdgcn_readlane(r.row, l);
      run.n = __builtin_amdgcn_readlane(r.n, l);
      run.pos = __builtin_amdgcn_readlane(r.pos, l);
      page = u - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l));
      return b0 + l;
    }
    base = __builtin_amdgcn_readlane(upto, 63);
  }
  return -1;
}

constexpr int kAppendThreads = 128;

// One workgroup per (page of a sequence's run, KV head) stores the page's new
// keys (token-major) and values (d-major, transposed through LDS, whole 16-byte
// pieces where the run covers them) and widens the digest; as many others turn
// the queries of the page's rows, G heads each.  The positions come from
// start_pos, so that one workgroup can advance seq_lens while the others run.
template <typename T, int PS, int D>
__global__ void __launch_bounds__(kAppendThreads) append_rotary_kernel(
    Geometry g, int step, retro_chunk ch, retro_rotary r, T* __restrict__ kc, T* __restrict__ vc,
    T* __restrict__ dg, const int32_t* __restrict__ pt, int32_t* __restrict__ seq_lens,
    int32_t* __restrict__ loaded, const T* q, int64_t q_stride, const T* __restrict__ k,
    int64_t k_stride, const T* __restrict__ v, int64_t v_stride, T* q_out) {
  using Tn = Turn<T, D>;
  constexpr int E = Tn::E, LPV = Tn::LPV;
  constexpr int ROW = D + E;  // padded LDS row
  __shared__ __attribute__((aligned(16))) T ks[PS * ROW];
  __shared__ __attribute__((aligned(16))) T vs[PS * ROW];
  __shared__ int first_bad;
  const int tid = threadIdx.x, lane = tid & 63;
  Run run;
  int page;
  // a page's workgroups are neighbours on one XCD: they read and write neighbouring
  // memory, and the same angles (21828 rows, 554 MB: 142 us as a row of all pages for
  // each head, 129 as neighbours on all XCDs, 119 on one)
  const int kinds = q ? 2 * g.hk : g.hk, i = blockIdx.x >> 3, kind = i % kinds;
  const int b = find_page(ch, g.batch, PS, lane, i / kinds * 8 + (blockIdx.x & 7), run, page);
  if (b < 0 || page < 0 || page >= run_pages(run, PS)) return;
  const int lp0 = run.pos / PS, lp = lp0 + page;
  // slots of this page that the run fills, and the row of slot 0
  const int s0 = page ? 0 : run.pos - lp * PS;
  const int s1 = (int)min((int64_t)PS, (int64_t)run.pos + run.n - (int64_t)lp * PS);
  const int64_t row0 = (int64_t)run.row + (int64_t)lp * PS - run.pos;
  const Tn turn(r, lane);
  typename Tn::Angles a;
  typename Tn::Weights wt;

  if (kind >= g.hk) {  // queries
    const int h0 = (kind - g.hk) * g.G;
    turn.weights(r.q_norm, wt);
    constexpr int AHEAD = 4;  // heads of a row on the way together
    for (int t = s0 + tid / LPV; t < s1; t += kAppendThreads / LPV) {
      turn.angles(lp * PS + t, a);
      for (int g0 = 0; g0 < g.G; g0 += AHEAD) {
        u32x4 raw[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
          raw[i] = reinterpret_cast<const u32x4*>(q + (row0 + t) * q_stride +
                                                  (h0 + min(g0 + i, g.G - 1)) * D)[turn.c];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
          if (g0 + i < g.G)
            reinterpret_cast<u32x4*>(q_out + ((row0 + t) * g.hq + h0 + g0 + i) * D)[turn.c] =
                turn(raw[i], r.q_norm != nullptr, wt, a, lane);
      }
    }
    return;
  }

  const int h = kind;
  if (page == 0 && h == 0) {  // the sequence's new length: up to its first page that is not mapped
    const int np = run_pages(run, PS);
    if (tid == 0) first_bad = np;
    __syncthreads();
    for (int i = tid; i < np; i += kAppendThreads) {
      const int ph = lp0 + i < g.max_pages ? pt[(int64_t)b * g.max_pages + lp0 + i] : -1;
      if (ph < 0 || ph >= g.num_phys) {
        atomicMin(&first_bad, i);
        break;
      }
    }
    __syncthreads();
    if (tid == 0 && first_bad > 0)
      seq_lens[b] = (int)min((int64_t)run.pos + run.n, (int64_t)(lp0 + first_bad) * PS);
  }
  if (lp >= g.max_pages) return;
  const int phys = pt[(int64_t)b * g.max_pages + lp];
  if (phys < 0 || phys >= g.num_phys) return;
  const int64_t blk = ((int64_t)phys * g.hk + h) * PS * D;
  turn.weights(r.k_norm, wt);
  constexpr int NP = PS * LPV / kAppendThreads;  // passes over a page's rows
  u32x4 kr[NP], vr[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int t = tid / LPV + i * (kAppendThreads / LPV);
    if (t < s0 || t >= s1) continue;
    kr[i] = reinterpret_cast<const u32x4*>(k + (row0 + t) * k_stride + h * D)[turn.c];
    vr[i] = reinterpret_cast<const u32x4*>(v + (row0 + t) * v_stride + h * D)[turn.c];
  }
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int t = tid / LPV + i * (kAppendThreads / LPV);
    if (t < s0 || t >= s1) continue;
    turn.angles(lp * PS + t, a);
    const u32x4 kt = turn(kr[i], r.k_norm != nullptr, wt, a, lane);
    reinterpret_cast<u32x4*>(kc + blk + t * D)[turn.c] = kt;
    *reinterpret_cast<u32x4*>(ks + t * ROW + turn.c * E) = kt;
    *reinterpret_cast<u32x4*>(vs + t * ROW + turn.c * E) = vr[i];
  }
  __syncthreads();
  // values: E consecutive tokens of one element of d per piece
  for (int e = tid; e < D * (PS / E); e += kAppendThreads) {
    const int i = e / (PS / E), t0 = e % (PS / E) * E;
    if (t0 + E <= s0 || t0 >= s1) continue;
    T* dst = vc + blk + (int64_t)i * PS + t0;
    T x[E];
#pragma unroll
    for (int j = 0; j < E; ++j) x[j] = vs[(t0 + j) * ROW + i];
    if (t0 >= s0 && t0 + E <= s1) {
      u32x4 u;
      __builtin_memcpy(&u, x, 16);
      *reinterpret_cast<u32x4*>(dst) = u;
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (t0 + j >= s0 && t0 + j < s1) dst[j] = x[j];
    }
  }
  T* drow = dg + ((((int64_t)b * g.hk + h) * g.max_pages + lp) * 2) * D;
  for (int i = tid; i < D; i += kAppendThreads) {
    T lo = s0 ? drow[i] : ks[i], hi = s0 ? drow[D + i] : ks[i];
    for (int t = s0; t < s1; ++t) {
      const T x = ks[t * ROW + i];
      if (to_f32(x) < to_f32(lo)) lo = x;
      if (to_f32(hi) < to_f32(x)) hi = x;
    }
    drow[i] = lo;
    drow[D + i] = hi;
  }
  if (tid == 0) loaded[((int64_t)b * g.hk + h) * g.max_pages + lp] = step - 1;
}

// f(type, head_dim) for the dims' type and head size
template <typename F>
auto with_type_and_dim(const Geometry& g, F f) {
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (g.dtype == RETRO_BF16) return g.D == 128 ? f(bf16_t{}, D128{}) : f(bf16_t{}, D64{});
  return g.D == 128 ? f(float{}, D128{}) : f(float{}, D64{});
}

// Groups of heads per wavefront: one where there are few rows (64 rows of 40 heads: 4.0
// us), five where the wavefronts fill the GPU many times over (8192 rows of 40 heads, 172
// MB: 60 us with one, 54, 52, 49, 48 and 48 with 2, 3, 4, 5 and 8; 36.5 us, 4.7 TB/s, with
// the outputs written past the L2s).
constexpr int kManyGroups = 5;
int rotate_groups(const Geometry& g, int rows, bool q, bool k) {
  const int64_t vpw = 64 / (g.D * g.elt / 16), heads = (q ? g.hq : 0) + (int64_t)(k ? g.hk : 0);
  return rows * ((heads + vpw - 1) / vpw) > 16384 ? kManyGroups : 1;
}
int64_t rotate_blocks(const Geometry& g, int rows, bool q, bool k) {
  const int64_t vpw = 64 / (g.D * g.elt / 16) * rotate_groups(g, rows, q, k);
  const int64_t heads = (q ? g.hq : 0) + (int64_t)(k ? g.hk : 0);
  return (rows * ((heads + vpw - 1) / vpw) + 3) / 4;
}

// every sequence's pages, at most n / P + 2 of each, in eights (an XCD's workgroups are
// every eighth), times the workgroups of a page
int64_t append_blocks(const Geometry& g, int n_rows, bool q) {
  const int64_t pages = n_rows / g.P + 2 * (int64_t)std::min(g.batch, n_rows);
  return (pages + 7) / 8 * 8 * (q ? 2 : 1) * g.hk;
}

}  // namespace

hipError_t launch_rotary_table(float* table, int positions, int rot_dim, double base, hipStream_t s) {
  const int64_t n = (int64_t)positions * (rot_dim / 2);
  rotary_table_kernel<<<(unsigned)std::min<int64_t>((n + 255) / 256, 8192), 256, 0, s>>>(
      table, n, rot_dim / 2, rot_dim, log2(base));
  return hipGetLastError();
}

bool rotate_qk_supported(const Geometry& g, int rows, bool q, bool k) {
  // (the last workgroup's wavefronts go up to three rows past the last one)
  return rotate_blocks(g, rows, q, k) < (int64_t)1 << 31 && rows < 0x7fffffff - 3;
}

hipError_t launch_rotate_qk(const Geometry& g, const retro_rotary& r, const int32_t* positions,
                            int rows, const void* q, int64_t q_stride, const void* k,
                            int64_t k_stride, void* q_out, void* k_out, hipStream_t s) {
  return with_type_and_dim(g, [&](auto t, auto d) {
    using T = decltype(t);
    auto go = [&](auto iter) {
      rotate_qk_kernel<T, decltype(d)::value, decltype(iter)::value>
          <<<(unsigned)rotate_blocks(g, rows, q, k), 256, 0, s>>>(
              r, positions, rows, q ? g.hq : 0, k ? g.hk : 0, (const T*)q, q_stride, (const T*)k,
              k_stride, (T*)q_out, (T*)k_out);
      return hipGetLastError();
    };
    return rotate_groups(g, rows, q, k) == 1 ? go(std::integral_constant<int, 1>{})
                                             : go(std::integral_constant<int, kManyGroups>{});
  });
}

bool append_rotary_supported(const Geometry& g, int n_rows) {
  return append_blocks(g, n_rows, true) < (int64_t)1 << 31;
}

hipError_t launch_append_rotary(const Geometry& g, int step, const retro_kv_cache& c,
                                const retro_chunk& ch, const retro_rotary& r, const void* q,
                                int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                int64_t v_stride, void* q_out, hipStream_t s) {
  const unsigned grid = (unsigned)append_blocks(g, ch.n_rows, q != nullptr);
  return with_type_and_dim(g, [&](auto t, auto d) {
    using T = decltype(t);
    auto go = [&](auto ps) {
      append_rotary_kernel<T, decltype(ps)::value, decltype(d)::value><<<grid, kAppendThreads, 0, s>>>(
          g, step, ch, r, (T*)c.k_cache, (T*)c.v_cache, (T*)c.digest, c.page_table, c.seq_lens,
          c.last_loaded, (const T*)q, q_stride, (const T*)k, k_stride, (const T*)v, v_stride,
          (T*)q_out);
      return hipGetLastError();
    };
    return g.P == 16 ? go(std::integral_constant<int, 16>{}) : go(std::integral_constant<int, 32>{});
  });
}

}  // namespace retro
