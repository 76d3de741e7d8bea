// Attention of the retrospective window's queries over the selected pages of a cache in
// 4 bits: one (sequence, KV head, split, row group of RT tiles of 16) per workgroup, whose
// eight wavefronts take the split's chunks of 32 tokens in turn, straight from the pages
// into registers (mx4_rows.h), the next chunk's codes under way while one is worked on.
// A past query takes the pages with M_p < tau (Alg. 2, "Retrospective Mask" paragraph).
// The wavefronts' states are merged through LDS; the partial outputs and log-normalisers of
// a split go to the workspace as those of the other attention kernels, for the same
// combine launch, or where there is one split to the results themselves.
#include <algorithm>

#include "mx4_rows.h"

namespace retro {
namespace {

constexpr int kWaves = 8;
constexpr int kListPages = 512;  // pages of a split (list in LDS)

struct WindowCall {
  Geometry g;
  int step;
  const void *q, *kc, *vc;
  const int32_t *pt, *seq_lens, *sel, *msk, *nsel;
  float *o_ws, *l_ws;   // partials, or
  float *o_out, *l_out;  // the results, of a single split
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

template <typename T, int D, int P, int RT>
__global__ void __launch_bounds__(64 * kWaves, RT == 1 && sizeof(T) == 2 ? 4 : 2) mx4_window_kernel(WindowCall a) {
  constexpr int PT = 32 / P;  // pages of a chunk
  __shared__ __attribute__((aligned(16))) WindowLds<D, RT> L;
  const Geometry& g = a.g;
  const int tid = thread_index(), lane = tid & 63, ln16 = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // row group fastest: a split's row groups run at the same time on one XCD
  int u = xcd_remap(blockIdx.x, gridDim.x);
  const int rg = u % g.n_rgroups;
  u /= g.n_rgroups;
  const int split = u % g.n_splits;
  u /= g.n_splits;
  const int h = u % g.hk, b = u / g.hk, bh = b * g.hk + h, W = g.W;

  // the split's pages
  const int first = split * g.pages_per_split;
  const int rows_of_list = max(0, min(g.pages_per_split, g.k_max - first));
  const int np = min(rows_of_list, max(sload(a.nsel + bh) - first, 0));
  const int nch = (np + PT - 1) / PT, seq_len = sload(a.seq_lens + b);
  for (int i = tid; i < (rows_of_list + PT - 1) / PT * PT; i += 64 * kWaves) {
    // (entries behind the selected ones are read too, so as not to wait for their number)
    const int64_t o = (int64_t)bh * g.k_max + first + min(i, rows_of_list - 1);
    const int lp = a.sel[o], m = a.msk[o];
    const int phys = lp >= 0 && lp < g.max_pages ? a.pt[(int64_t)b * g.max_pages + lp] : -1;
    const bool ok = i < np && phys >= 0 && phys < g.num_phys;
    // a page without stored tokens reads page 0 of the pool; none of it is used
    L.list.phys[i] = ok ? phys : 0;
    L.list.len[i] = ok ? max(0, min(P, seq_len - lp * P)) : 0;
    L.list.mask[i] = m;
  }

  // the rows, and the mask value from which one may not use a page (none for a row
  // that does not exist, all for the current query)
  // (weights as three bf16 terms: the outputs are fp32 and merged again and again; with two, as
  // for chunks, they are 1.5e-6 off 64 bits instead of 1.5e-7, 128 heads of 36 rows 14.5 us
  // instead of 15.7)
  Mx4Rows<T, D, RT, 3> rows;
  rows.c = g.sm_scale * kLog2e;
  int thr[RT];
#pragma unroll
  for (int n = 0; n < RT; ++n) {
    const int rho = (rg * RT + n) * 16 + ln16;
    const bool live = rho < g.R;
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
  // Chunks are under way in two sets of registers in turn, or, with one tile of rows (and so
  // two workgroups on a compute unit), into the one as its keys, and then its values, are done with.
  constexpr int DEPTH = RT == 1 ? 1 : 2;
  auto work = [&](Mx4Tile<D>& x, int ch) {
    [[maybe_unused]] const int next = min(ch + kWaves, nch - 1);
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
        [&]() {
          if constexpr (DEPTH == 1) load_keys(x, next);
        },
        [&]() {
          if constexpr (DEPTH == 1) load_values(x, next);
        });
  };
  if (wave < nch) {
    Mx4Tile<D> x;
    int ch = wave;
    load_keys(x, ch);
    load_values(x, ch);
    if constexpr (DEPTH == 1) {
      for (; ch < nch; ch += kWaves) work(x, ch);
    } else {
      Mx4Tile<D> y;
      for (;;) {
        const bool more = ch + kWaves < nch;
        if (more) {
          load_keys(y, ch + kWaves);
          load_values(y, ch + kWaves);
        }
        work(x, ch);
        if (!more) break;
        ch += kWaves;
        const bool again = ch + kWaves < nch;
        if (again) {
          load_keys(x, ch + kWaves);
          load_values(x, ch + kWaves);
        }
        work(y, ch);
        if (!again) break;
        ch += kWaves;
      }
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
  // where row rho's outputs go, in rows of d
  auto place = [&](int rho) {
    const int r = rho / g.G;
    return a.o_out ? ((int64_t)b * (W + 1) + r) * g.hq + h * g.G + rho - r * g.G : part0 + rho;
  };
  float *const o_to = a.o_out ? a.o_out : a.o_ws, *const l_to = a.o_out ? a.l_out : a.l_ws;
#pragma unroll
  for (int n = 0; n < RT; ++n) {
    const int rho0 = (rg * RT + n) * 16, rr = n * 16 + ln16;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, L.m[w][rr]);
    const float Mu = M == -INFINITY ? 0.f : M;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      sum += L.l[w][rr] * __builtin_amdgcn_exp2f((L.m[w][rr] - Mu) * rows.c);
    // (a NaN sum, from NaN or infinite scores, makes the row NaN: here, or, with a
    // log-normaliser of +inf, in the combine)
    const float f = sum == 0.f ? 0.f : __builtin_amdgcn_exp2f((rows.m[n] - Mu) * rows.c) / sum;
    if (wave == 0 && quarter == 0 && rho0 + ln16 < g.R) {
      const float z = __builtin_fmaf(M, g.sm_scale, __log2f(sum) * kLn2);
      l_to[place(rho0 + ln16)] = a.o_out ? z : fminf(z, INFINITY);  // (fminf skips NaN)
    }
    if (n > 0) __syncthreads();  // the previous tile has been read
    rows.each(n, lane, [&](int d, f32x4 o) { *reinterpret_cast<f32x4*>(&L.o[wave][ln16][d]) = o * f; });
    __syncthreads();
    constexpr int VPR = D / 4;  // 16-byte pieces per row
    for (int e = tid; e < 16 * VPR; e += 64 * kWaves) {
      const int rw = e / VPR, c4 = (e - rw * VPR) * 4;
      f32x4 o = *reinterpret_cast<const f32x4*>(&L.o[0][rw][c4]);
#pragma unroll
      for (int w = 1; w < kWaves; ++w) o += *reinterpret_cast<const f32x4*>(&L.o[w][rw][c4]);
      if (rho0 + rw < g.R)
        __builtin_nontemporal_store(o, reinterpret_cast<f32x4*>(o_to + place(rho0 + rw) * D + c4));
    }
  }
}

template <typename T, int D, int P, int RT>
hipError_t go(const WindowCall& a, hipStream_t s) {
  const Geometry& g = a.g;
  const int64_t n = (int64_t)g.n_splits * g.n_rgroups * g.hk * g.batch;
  mx4_window_kernel<T, D, P, RT><<<(unsigned)n, 64 * kWaves, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T, int D, int P>
hipError_t go_tiles(const WindowCall& a, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (a.g.tiles_per_group == 2) return go<T, D, P, 2>(a, s);
  }
  return a.g.tiles_per_group == 1 ? go<T, D, P, 1>(a, s) : hipErrorInvalidValue;
}

}  // namespace

// One workgroup takes one or two tiles of rows (fp32 rows, with three times the operands, one)
// and a number of chunks that its wavefronts go through in `it` turns.  A turn takes 1.05 us
// with one tile and 1.95 with two (d 128), the beginning and end of two tiles 0.3 more than those
// of one, a further round of workgroups on a compute unit 1.2 and 4.7 (those of one tile are two
// at a time); splits cost a combine of 2.8 us and its partials, 0.54 us a million elements.
// These are fitted to 3724 draws of bf16 shapes (3159 different ones, d 64 and 128 together), each
// measured with one to three tiles in 1, 2, 4 .. 32 splits, and serve fp32 as they are.  On other draws, the
// choice among those splits is behind the best one of its shape by (mean, most) 0.5 and 31 %
// for bf16 of d 128 (1031 draws), 1.4 and 24 % of d 64 (462), fp32 0.7 and 16 % of d 128 (1524), 0.5 and 13 %
// of d 64 (709).  Three tiles a workgroup were the best of 99 of 3724 draws, by 4 % on average and
// 12 % at most (d 64, one split), which is 0.1 % over all, and have no kernel.
// Some choices: 16 heads of 68 rows, 128 pages, one tile in 3 splits 11.8 us (in 2 13.2, in 4 14.3,
// in one 15.2); 128 heads of 36 rows, 64 pages, two tiles in one 16.2 (one tile 16.8); 512 heads
// of 36 rows, 32 pages, one tile 29.0 (two 41.7, three 34.5).
Geometry mx4_window_geometry(const Geometry& g) {
  static constexpr float kTurn[2] = {1.05f, 1.95f}, kRound[2] = {1.2f, 4.7f}, kFirst[2] = {0.f, 0.3f};
  Geometry x = g;
  x.stream = 1;
  const int most = g.dtype == RETRO_BF16 ? 2 : 1, cap = compute_units(), cps_max = kListPages / g.chunk_pages;
  const float partial = 0.54e-6f * (float)((int64_t)g.batch * g.hq * (g.W + 1) * g.D);
  float best = 0.f;
  for (int rt = 1; rt <= std::min(most, g.row_tiles); ++rt) {
    const int groups = (g.row_tiles + rt - 1) / rt;
    for (int it = 1; it <= (std::min(g.chunks_max, cps_max) + kWaves - 1) / kWaves; ++it) {
      const int cps = std::min(it * kWaves, cps_max), ns = (g.chunks_max + cps - 1) / cps;
      if (ns > g.n_splits) continue;
      const int64_t rounds = ((int64_t)g.batch * g.hk * groups * ns + cap - 1) / cap;
      const float time = (float)(rounds * it) * kTurn[rt - 1] + (float)(rounds - 1) * kRound[rt - 1] +
                         kFirst[rt - 1] + (ns > 1 ? 2.8f + partial * (float)ns : 0.f);
      if (best != 0.f && time >= best) continue;
      best = time;
      x.tiles_per_group = rt;
      x.n_rgroups = groups;
      x.chunks_per_split = (g.chunks_max + ns - 1) / ns;
    }
  }
  x.n_splits = (g.chunks_max + x.chunks_per_split - 1) / x.chunks_per_split;
  x.pages_per_split = x.chunks_per_split * g.chunk_pages;
  return x;
}

hipError_t launch_mx4_window(const Geometry& g, int step, const void* q_window, const retro_kv_cache& c,
                             const retro_selection& sel, float* o_ws, float* l_ws, float* o_out, float* l_out,
                             hipStream_t s) {
  const WindowCall a{g,           step,         q_window, c.k_cache,        c.v_cache, c.page_table,
                     c.seq_lens,  sel.selected, sel.mask, sel.num_selected, o_ws,      l_ws,
                     o_out,       l_out};
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
