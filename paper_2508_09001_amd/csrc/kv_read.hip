// Rows of the paged cache as keys and values again, whatever the cache's format: a copy
// out of the pages, in 4 bits with the codes' values.
//
// One workgroup per (page of a sequence's run, KV head), a page's as neighbours on one
// XCD, as in the append.  Bound by HBM: every code is read once and every value written
// once (32768 rows of 8 KV heads of 128 out of 4 bits, 170 MB, 26.2 us, 6.5 TB/s; 39.3 with the values
// kept in the L2s).
#include "mx4.h"
#include "rotary.h"

namespace retro {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kReadThreads = 128;
constexpr int64_t kL2Bytes = 32 << 20;

// PAST: the values are more than the L2s hold and are written past them.
template <typename T, int PS, int D, bool MX4, bool PAST>
__global__ void __launch_bounds__(kReadThreads) read_kv_kernel(Geometry g, retro_chunk ch,
                                                               const char* __restrict__ kc,
                                                               const char* __restrict__ vc,
                                                               const int32_t* __restrict__ pt,
                                                               const int32_t* __restrict__ seq_lens,
                                                               T* __restrict__ k_out, T* __restrict__ v_out) {
  constexpr int E = 16 / sizeof(T), LPV = D / E, NP = PS * LPV / kReadThreads;
  constexpr int ROW = D + E;  // padded LDS row
  __shared__ __attribute__((aligned(16))) T vs[MX4 ? E : PS * ROW];
  const int tid = threadIdx.x, i = blockIdx.x >> 3, h = i % g.hk;
  Run run;
  int page;
  const int b = find_page(ch, g.batch, PS, tid & 63, i / g.hk * 8 + (blockIdx.x & 7), run, page);
  if (b < 0 || page < 0 || page >= run_pages(run, PS)) return;
  const int lp = run.pos / PS + page;
  const int s0 = page ? 0 : run.pos - lp * PS;
  const int s1 = (int)min((int64_t)PS, (int64_t)run.pos + run.n - (int64_t)lp * PS);
  const int64_t row0 = (int64_t)run.row + (int64_t)lp * PS - run.pos;
  // slots that hold a token
  const int phys = lp < g.max_pages ? pt[(int64_t)b * g.max_pages + lp] : -1;
  const int held = phys >= 0 && phys < g.num_phys
                       ? (int)min(max((int64_t)seq_lens[b] - (int64_t)lp * PS, (int64_t)0), (int64_t)PS)
                       : 0;
  constexpr int kBytes = MX4 ? mx4_block_bytes(PS, D) : PS * D * (int)sizeof(T);
  const int64_t block = (int64_t)max(phys, 0) * g.hk + h;
  const char *kblk = kc + block * kBytes, *vblk = vc + block * kBytes;
  const int c = tid % LPV;
  auto put = [](T* to, u32x4 x) {
    if constexpr (PAST) __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(to));
    else *reinterpret_cast<u32x4*>(to) = x;
  };
  if constexpr (MX4) {
    uint32_t code[2][NP];
    int e[2][NP];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int t = tid / LPV + j * (kReadThreads / LPV);
      code[0][j] = code[1][j] = 0;
      e[0][j] = e[1][j] = 127;
      if (t < s0 || t >= min(s1, held)) continue;
      const int at_block = c * E / 32;
      if (k_out) {
        const char* p = kblk + t * (D / 2) + c * (E / 2);
        code[0][j] = E == 8 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
        e[0][j] = (uint8_t)kblk[PS * D / 2 + t * (D / 32) + at_block];
      }
      if (v_out) {
        const char* group = vblk + t / 4 * (2 * D);
        const int part = c * E / (D / 16), in = c * E % (D / 16);
        if constexpr (E > D / 16) {  // two parts of four elements
          const uint16_t* p = reinterpret_cast<const uint16_t*>(group) + part * 4 + t % 4;
          code[1][j] = p[0] | (uint32_t)p[4] << 16;
        } else {
          const char* p = group + (part * 4 + t % 4) * (D / 32) + in / 2;
          code[1][j] = E == 8 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
        }
        e[1][j] = (uint8_t)vblk[PS * D / 2 + (t / 4 * (D / 32) + at_block) * 4 + t % 4];
      }
    }
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int t = tid / LPV + j * (kReadThreads / LPV);
      if (t < s0 || t >= s1) continue;
      const int64_t at = ((row0 + t) * g.hk + h) * D + c * E;
      if (k_out) put(k_out + at, mx4_piece<T>(code[0][j], mx4_scale(e[0][j])));
      if (v_out) put(v_out + at, mx4_piece<T>(code[1][j], mx4_scale(e[1][j])));
    }
  } else {
    if (v_out) {  // E consecutive tokens of one element of d per piece
      for (int e = tid; held && e < D * (PS / E); e += kReadThreads) {
        const int i = e / (PS / E), t0 = e % (PS / E) * E;
        const u32x4 x = reinterpret_cast<const u32x4*>(vblk)[e];
        T v[E];
        __builtin_memcpy(v, &x, 16);
#pragma unroll
        for (int j = 0; j < E; ++j) vs[(t0 + j) * ROW + i] = v[j];
      }
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int t = tid / LPV + j * (kReadThreads / LPV);
      if (t < s0 || t >= s1) continue;
      const int64_t at = ((row0 + t) * g.hk + h) * D + c * E;
      u32x4 k{0, 0, 0, 0}, v{0, 0, 0, 0};
      if (t < held && k_out) k = reinterpret_cast<const u32x4*>(kblk)[t * LPV + c];
      if (t < held && v_out) v = *reinterpret_cast<const u32x4*>(vs + t * ROW + c * E);
      if (k_out) put(k_out + at, k);
      if (v_out) put(v_out + at, v);
    }
  }
}

}  // namespace

bool read_kv_supported(const Geometry& g, int n_rows) { return page_blocks(g, n_rows, g.hk) < (int64_t)1 << 31; }

hipError_t launch_read_kv(const Geometry& g, const retro_kv_cache& c, const retro_chunk& ch, void* k_out,
                          void* v_out, hipStream_t s) {
  const unsigned grid = (unsigned)page_blocks(g, ch.n_rows, g.hk);
  const bool past = (int64_t)ch.n_rows * g.hk * g.D * g.elt * ((k_out != nullptr) + (v_out != nullptr)) > kL2Bytes;
  auto launch = [&](auto t, auto ps, auto d, auto in_4_bits, auto past_l2) {
    using T = decltype(t);
    read_kv_kernel<T, decltype(ps)::value, decltype(d)::value, decltype(in_4_bits)::value, decltype(past_l2)::value>
        <<<grid, kReadThreads, 0, s>>>(g, ch, (const char*)c.k_cache, (const char*)c.v_cache, c.page_table,
                                       c.seq_lens, (T*)k_out, (T*)v_out);
    return hipGetLastError();
  };
  auto go = [&](auto t, auto ps, auto d, auto in_4_bits) {
    return past ? launch(t, ps, d, in_4_bits, std::true_type{}) : launch(t, ps, d, in_4_bits, std::false_type{});
  };
  auto with_format = [&](auto t, auto ps, auto d) {
    return is_mx4(g) ? go(t, ps, d, std::true_type{}) : go(t, ps, d, std::false_type{});
  };
  auto with_d = [&](auto t, auto ps) {
    return g.D == 128 ? with_format(t, ps, std::integral_constant<int, 128>{})
                      : with_format(t, ps, std::integral_constant<int, 64>{});
  };
  auto with_page = [&](auto t) {
    return g.P == 16 ? with_d(t, std::integral_constant<int, 16>{}) : with_d(t, std::integral_constant<int, 32>{});
  };
  return g.dtype == RETRO_BF16 ? with_page(bf16_t{}) : with_page(float{});
}

}  // namespace retro
