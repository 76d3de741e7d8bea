// Attention of the retrospective window's queries over the selected pages of a cache in
// 4 bits: one (sequence, KV head, split, row group) per workgroup, its eight wavefronts
// SIDE side by side over the rows (RT tiles of 16 each) and NT = 8 / SIDE over the
// split's chunks of 32 tokens (wt, wt + NT, ...), which they read straight from the pages
// into registers (mx4_rows.h), the next chunk's codes under way while one is worked on.
// A past query takes the pages with M_p < tau (Alg. 2, "Retrospective Mask" paragraph).
// The wavefronts' states are merged through LDS; the partial outputs and log-normalisers of
// a split go to the workspace as those of the other attention kernels, for the same
// combine launch.
#include <algorithm>

#include "mx4_rows.h"

namespace retro {
namespace {

constexpr int kWaves = 8;
constexpr int kListPages = 1024;  // pages of a split (list in LDS)

struct WindowCall {
  Geometry g;
  int step;
  const void *q, *kc, *vc;
  const int32_t *pt, *seq_lens, *sel, *msk, *nsel;
  float *o_ws, *l_ws;
};

template <int D, int RT>
struct WindowLds {
  static constexpr int OROW = D + 4;
  struct {
    int phys[kListPages], len[kListPages], mask[kListPages];
  } list;
  float o[kWaves][16][OROW];
  float m[kWaves][RT * 16], l[kWaves][RT * 16];
};

template <typename T, int D, int P, int RT, int SIDE>
__global__ void __launch_bounds__(64 * kWaves) mx4_window_kernel(WindowCall a) {
  constexpr int NT = kWaves / SIDE, PT = 32 / P;  // pages of a chunk
  __shared__ __attribute__((aligned(16))) WindowLds<D, RT> L;
  const Geometry& g = a.g;
  const int tid = thread_index(), lane = tid & 63, ln16 = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % SIDE, wt = wave / SIDE;
  // row group fastest: a split's row groups run at the same time on one XCD
  int u = xcd_remap(blockIdx.x, gridDim.x);
  const int rg = u % g.n_rgroups;
  u /= g.n_rgroups;
  const int split = u % g.n_splits;
  u /= g.n_splits;
  const int h = u % g.hk, b = u / g.hk, bh = b * g.hk + h, W = g.W;

  // the split's pages
  const int first = split * g.pages_per_split;
  const int np = max(0, min(min(g.pages_per_split, a.nsel[bh] - first), g.k_max - first));
  const int nch = (np + PT - 1) / PT;
  const int seq_len = a.seq_lens[b];
  for (int i = tid; i < nch * PT; i += 64 * kWaves) {
    int lp = -1, m = 0, phys = -1;
    if (i < np) {
      const int64_t o = (int64_t)bh * g.k_max + first + i;
      lp = a.sel[o];
      m = a.msk[o];
      if (lp >= 0 && lp < g.max_pages) phys = a.pt[(int64_t)b * g.max_pages + lp];
    }
    const bool ok = phys >= 0 && phys < g.num_phys;
    // a page without stored tokens reads page 0 of the pool; none of it is used
    L.list.phys[i] = ok ? phys : 0;
    L.list.len[i] = ok ? max(0, min(P, seq_len - lp * P)) : 0;
    L.list.mask[i] = m;
  }

  // the rows, and the mask value from which one may not use a page (none for a row
  // that does not exist, all for the current query)
  Mx4Rows<T, D, RT> rows;
  rows.c = g.sm_scale * kLog2e;
  int thr[RT];
#pragma unroll
  for (int n = 0; n < RT; ++n) {
    const int lt = wr * RT + n, rho = (rg * g.tiles_per_group + lt) * 16 + ln16;
    const bool live = lt < g.tiles_per_group && rho < g.R;
    const int r = live ? rho / g.G : 0, gq = live ? rho - r * g.G : 0, tau = a.step - W + r;
    thr[n] = (live && tau >= 0) ? (r == W ? 0x7fffffff : tau) : (int)0x80000000;
    rows.start(n, (const T*)a.q + (((int64_t)b * (W + 1) + r) * g.hq + (int64_t)h * g.G + gq) * D, live, lane);
  }
  __syncthreads();

  constexpr int64_t kBlock = mx4_block_bytes(P, D);
  const Mx4Places<D, P> at(lane);
  const char* kh = (const char*)a.kc + h * kBlock;
  const char* vh = (const char*)a.vc + h * kBlock;
  auto block = [&](int ch, int t) {
    return (int64_t)__builtin_amdgcn_readfirstlane(L.list.phys[ch * PT + (PT == 2 ? t : 0)]) * (kBlock * g.hk);
  };
  auto load_keys = [&](Mx4Tile<D>& x, int ch) {
#pragma unroll
    for (int t = 0; t < 2; ++t) at.template load_keys<false>(x, t, kh + block(ch, t), PT == 2 ? 0 : 16 * t);
  };
  auto load_values = [&](Mx4Tile<D>& x, int ch) {
#pragma unroll
    for (int t = 0; t < 2; ++t) at.template load_values<false>(x, t, vh + block(ch, t), PT == 2 ? 0 : 16 * t);
  };
  auto work = [&](Mx4Tile<D>& x, int ch) {
    int live[2], mask[2];  // of the lane's four tokens of each half
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int slot = ch * PT + (PT == 2 ? t : 0);
      live[t] = L.list.len[slot] - (PT == 2 ? 0 : 16 * t) - 4 * quarter;
      mask[t] = L.list.mask[slot];
    }
    const bool cut = wave_ballot(min(live[0], live[1]) < 4) != 0;
    if (cut)
#pragma unroll
      for (int t = 0; t < 2; ++t) x.ve[t] = live_exponents(x.ve[t], live[t]);
    rows.step(
        x,
        [&](int n, f32x4(&s)[2]) {
          if (!cut && wave_ballot(max(mask[0], mask[1]) >= thr[n]) == 0) return;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e >= live[t] || mask[t] >= thr[n]) s[t][e] = -INFINITY;
        },
        [] {}, [] {});
  };
  if (wt < nch) {
    Mx4Tile<D> x, y;
    int ch = wt;
    load_keys(x, ch);
    load_values(x, ch);
    for (;;) {
      const bool more = ch + NT < nch;
      if (more) {
        load_keys(y, ch + NT);
        load_values(y, ch + NT);
      }
      work(x, ch);
      if (!more) break;
      ch += NT;
      const bool again = ch + NT < nch;
      if (again) {
        load_keys(x, ch + NT);
        load_values(x, ch + NT);
      }
      work(y, ch);
      if (!again) break;
      ch += NT;
    }
  }

  // ---- merge the wavefronts' states: factors per row, then the outputs tile by tile
#pragma unroll
  for (int n = 0; n < RT; ++n) {
    const float l = col_sum4(rows.l[n]);
    if (lane < 16) {
      L.m[wave][n * 16 + lane] = rows.m[n];
      L.l[wave][n * 16 + lane] = l;
    }
  }
  __syncthreads();
  const int64_t part0 = ((int64_t)bh * g.n_splits + split) * g.R;
#pragma unroll
  for (int n = 0; n < RT; ++n) {
    const int lt = wr * RT + n, row = (rg * g.tiles_per_group + lt) * 16 + ln16, rr = n * 16 + ln16;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < NT; ++w) M = fmaxf(M, L.m[w * SIDE + wr][rr]);
    const float Mu = M == -INFINITY ? 0.f : M;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < NT; ++w)
      sum += L.l[w * SIDE + wr][rr] * __builtin_amdgcn_exp2f((L.m[w * SIDE + wr][rr] - Mu) * rows.c);
    const float f = sum > 0.f ? __builtin_amdgcn_exp2f((rows.m[n] - Mu) * rows.c) / sum : 0.f;
    // -inf for an empty sum; +inf (fminf skips NaN) for a NaN one, from NaN or infinite
    // scores: the combine then makes the row NaN
    if (wt == 0 && quarter == 0 && lt < g.tiles_per_group && row < g.R)
      a.l_ws[part0 + row] = fminf(__builtin_fmaf(M, g.sm_scale, __log2f(sum) * kLn2), INFINITY);
    if (n > 0) __syncthreads();  // the previous tiles have been read
    rows.each(n, lane, [&](int d, f32x4 o) { *reinterpret_cast<f32x4*>(&L.o[wave][ln16][d]) = o * f; });
    __syncthreads();
    constexpr int VPR = D / 4;  // 16-byte pieces per row
    // tile n of each of the SIDE row ranges: the NT wavefronts' rows added up
#pragma unroll
    for (int r0 = 0; r0 < SIDE; ++r0) {
      const int t0 = r0 * RT + n;
      if (t0 >= g.tiles_per_group) break;  // uniform
      const int row0 = (rg * g.tiles_per_group + t0) * 16;
      for (int e = tid; e < 16 * VPR; e += 64 * kWaves) {
        const int rw = e / VPR, c4 = (e - rw * VPR) * 4;
        f32x4 o = *reinterpret_cast<const f32x4*>(&L.o[r0][rw][c4]);
#pragma unroll
        for (int w = 1; w < NT; ++w) o += *reinterpret_cast<const f32x4*>(&L.o[w * SIDE + r0][rw][c4]);
        if (row0 + rw < g.R)
          __builtin_nontemporal_store(o, reinterpret_cast<f32x4*>(a.o_ws + (part0 + row0 + rw) * D + c4));
      }
    }
  }
}

// tiles of 16 rows of a workgroup at most, and how its wavefronts share `tiles` of them:
// RT each, SIDE side by side.  (fp32 rows have three times the operands: a tile each.)
constexpr int most_tiles(int dtype) { return dtype == RETRO_BF16 ? 6 : 4; }
int side_by_side(int dtype, int tiles) {
  return dtype == RETRO_BF16 ? (tiles <= 3 ? 1 : 2) : (tiles == 1 ? 1 : tiles == 2 ? 2 : 4);
}

template <typename T, int D, int P, int RT, int SIDE>
hipError_t go(const WindowCall& a, hipStream_t s) {
  const Geometry& g = a.g;
  const int64_t n = (int64_t)g.n_splits * g.n_rgroups * g.hk * g.batch;
  mx4_window_kernel<T, D, P, RT, SIDE><<<(unsigned)n, 64 * kWaves, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T, int D, int P>
hipError_t go_tiles(const WindowCall& a, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    switch (a.g.tiles_per_group) {
      case 1: return go<T, D, P, 1, 1>(a, s);
      case 2: return go<T, D, P, 2, 1>(a, s);
      case 3: return go<T, D, P, 3, 1>(a, s);
      case 4: return go<T, D, P, 2, 2>(a, s);
      case 5:
      case 6: return go<T, D, P, 3, 2>(a, s);
      default: return hipErrorInvalidValue;
    }
  } else {
    switch (a.g.tiles_per_group) {
      case 1: return go<T, D, P, 1, 1>(a, s);
      case 2: return go<T, D, P, 1, 2>(a, s);
      case 3:
      case 4: return go<T, D, P, 1, 4>(a, s);
      default: return hipErrorInvalidValue;
    }
  }
}

}  // namespace

Geometry mx4_window_geometry(const Geometry& g) {
  Geometry x = g;
  const int most = most_tiles(g.dtype);
  x.n_rgroups = (g.row_tiles + most - 1) / most;
  x.tiles_per_group = (g.row_tiles + x.n_rgroups - 1) / x.n_rgroups;
  x.stream = 1;
  // the split count with the smallest time, counted in chunk iterations of a wavefront: rounds
  // of workgroups times the iterations of one, plus three for its start and merge
  const int nt = kWaves / side_by_side(g.dtype, x.tiles_per_group);
  const int64_t heads = (int64_t)g.batch * g.hk * x.n_rgroups;
  const int cap = compute_units(), cps_max = kListPages / g.chunk_pages;
  int best = 0;
  int64_t best_cost = 0;
  for (int it = (std::min(g.chunks_max, cps_max) + nt - 1) / nt; it >= 1; --it) {
    const int cps = std::min(it * nt, cps_max), ns = (g.chunks_max + cps - 1) / cps;
    if (ns > g.n_splits) break;
    const int64_t cost = (heads * ns + cap - 1) / cap * (it + 3);
    if (best == 0 || cost < best_cost) {
      best = ns;
      best_cost = cost;
    }
  }
  if (best == 0) best = g.n_splits;
  x.chunks_per_split = (g.chunks_max + best - 1) / best;
  x.n_splits = (g.chunks_max + x.chunks_per_split - 1) / x.chunks_per_split;
  x.pages_per_split = x.chunks_per_split * g.chunk_pages;
  return x;
}

hipError_t launch_mx4_window(const Geometry& g, int step, const void* q_window, const retro_kv_cache& c,
                             const retro_selection& sel, float* o_ws, float* l_ws, hipStream_t s) {
  const WindowCall a{g,          step,         q_window,         c.k_cache, c.v_cache, c.page_table, c.seq_lens,
                     sel.selected, sel.mask, sel.num_selected, o_ws,      l_ws};
  auto with_page = [&](auto t, auto d) {
    return g.P == 16 ? go_tiles<decltype(t), decltype(d)::value, 16>(a, s)
                     : go_tiles<decltype(t), decltype(d)::value, 32>(a, s);
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (g.dtype == RETRO_BF16) return g.D == 128 ? with_page(bf16_t{}, D128{}) : with_page(bf16_t{}, D64{});
  return g.D == 128 ? with_page(float{}, D128{}) : with_page(float{}, D64{});
}

}  // namespace retro
