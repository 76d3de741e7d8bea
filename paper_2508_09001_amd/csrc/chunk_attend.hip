// Dense causal attention of a ragged batch of rows over the paged cache.
#include "roles.h"
#include "rotary.h"

namespace retro {
namespace {

// One wavefront per (row, query head): 64 keys at a time, one per lane, and then
// the elements of d spread over the lanes.
template <typename T, int D>
__global__ void __launch_bounds__(64) chunk_attend_kernel(Geometry g, retro_chunk ch,
                                                          const T* __restrict__ kc,
                                                          const T* __restrict__ vc,
                                                          const int32_t* __restrict__ pt,
                                                          const int32_t* __restrict__ seq_lens,
                                                          const T* __restrict__ q, int64_t q_stride,
                                                          T* __restrict__ out,
                                                          float* __restrict__ lse) {
  __shared__ float sq[D], sp[64];
  __shared__ int sphys[64];
  const int lane = threadIdx.x, row = blockIdx.x, hq = blockIdx.y, h = hq / g.G;
  int b = 0;
  Run run{0, 0, 0};
  for (; b < g.batch; ++b) {
    run = chunk_run(ch, b);
    if (row >= run.row && row < run.row + run.n) break;
  }
  if (b == g.batch) return;
  const int p = run.pos + row - run.row;
  const int end = (int)min(min((int64_t)p + 1, (int64_t)seq_lens[b]), (int64_t)g.max_pages * g.P);
  for (int i = lane; i < D; i += 64) sq[i] = to_f32(q[row * q_stride + hq * D + i]);
  __syncthreads();
  float m = -INFINITY, l = 0.f, o[D / 64];
  for (int i = 0; i < D / 64; ++i) o[i] = 0.f;
  for (int k0 = 0; k0 < end; k0 += 64) {
    const int key = k0 + lane;
    int ph = key < end ? pt[(int64_t)b * g.max_pages + key / g.P] : -1;
    if (ph >= g.num_phys) ph = -1;
    float s = 0.f;
    if (ph >= 0)
      for (int i = 0; i < D; ++i)
        s += sq[i] * to_f32(kc[(((int64_t)ph * g.hk + h) * g.P + key % g.P) * D + i]);
    s = ph >= 0 ? s * g.sm_scale : -INFINITY;
    const float mn = fmaxf(m, wave_max(s)), mu = mn == -INFINITY ? 0.f : mn;
    const float e = ph >= 0 ? expf(s - mu) : 0.f, alpha = expf(m - mu);
    l = l * alpha + wave_sum(e);
    m = mn;
    sp[lane] = e;
    sphys[lane] = ph;
    __syncthreads();
    for (int i = 0; i < D / 64; ++i) o[i] *= alpha;
    for (int j = 0; j < 64; ++j) {
      if (sphys[j] < 0) continue;
      const T* vr = vc + ((int64_t)sphys[j] * g.hk + h) * g.P * D + (k0 + j) % g.P;
      for (int i = 0; i < D / 64; ++i) o[i] += sp[j] * to_f32(vr[(lane + i * 64) * g.P]);
    }
    __syncthreads();
  }
  const int64_t at = (int64_t)row * g.hq + hq;
  for (int i = 0; i < D / 64; ++i) {
    const float y = l == 0.f ? 0.f : o[i] / l;
    if constexpr (sizeof(T) == 2) {
      const __bf16 w = (__bf16)y;
      out[at * D + lane + i * 64].bits = __builtin_bit_cast(uint16_t, w);
    } else {
      out[at * D + lane + i * 64] = y;
    }
  }
  if (lse && lane == 0) lse[at] = l == 0.f ? -INFINITY : m + logf(l);
}

}  // namespace

bool chunk_attend_supported(const Geometry& g, int n_rows) {
  return (int64_t)n_rows * g.hq * g.D < (int64_t)1 << 40 && g.hq <= 65535;
}

size_t chunk_workspace(const Geometry&, int) { return 256; }

hipError_t launch_chunk_attend(const Geometry& g, const retro_kv_cache& c, const retro_chunk& ch,
                               const void* q, int64_t q_stride, void* out, float* lse, void*,
                               hipStream_t s) {
  const dim3 grid((unsigned)ch.n_rows, (unsigned)g.hq);
  auto go = [&](auto t, auto d) {
    using T = decltype(t);
    chunk_attend_kernel<T, decltype(d)::value><<<grid, 64, 0, s>>>(
        g, ch, (const T*)c.k_cache, (const T*)c.v_cache, c.page_table, c.seq_lens, (const T*)q,
        q_stride, (T*)out, lse);
    return hipGetLastError();
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (g.dtype == RETRO_BF16) return g.D == 128 ? go(bf16_t{}, D128{}) : go(bf16_t{}, D64{});
  return g.D == 128 ? go(float{}, D128{}) : go(float{}, D64{});
}

}  // namespace retro
