// KV storage of a cache in 4 bits without norms and rotations: AppendKV (Alg. 1), bulk
// prefill and UpdateKV, as kv_store.hip for a cache in dtype.  A head's vector is read as
// 16-byte pieces by consecutive lanes, which round a block together and write its codes
// to their places (mx4.h); digests are those of what the codes stand for.
#include <algorithm>

#include "mx4.h"

namespace retro {
namespace {

// Value i of token t of a page whose keys are at `block`.
template <int PS, int D>
__device__ __forceinline__ float stored_key(const char* block, int t, int i) {
  const uint32_t code = (uint8_t)block[t * (D / 2) + i / 2];
  const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(
      code, mx4_scale((uint8_t)block[PS * D / 2 + t * (D / 32) + i / 32]), 0);
  return i & 1 ? v[1] : v[0];
}
__device__ __forceinline__ void from_f32(float x, float* to) { *to = x; }
__device__ __forceinline__ void from_f32(float x, bf16_t* to) {
  to->bits = (uint16_t)(__float_as_uint(x) >> 16);  // exact: x is a bf16 value
}

// Tokens 0 .. n_tok - 1 (at most kMx4AppendTokens) of every sequence to its end, one
// workgroup per sequence: bound by the launch and four dependent round trips.  The first token whose
// page is not mapped is dropped with those behind it, as with the append in dtype.
constexpr int kMx4AppendTokens = 64;
constexpr int kAppendThreads = 1024;

template <typename T, int PS, int D>
__global__ void __launch_bounds__(kAppendThreads) mx4_append_kernel(
    Geometry g, int step, int n_tok, char* kc, char* __restrict__ vc, T* __restrict__ dg,
    const int32_t* __restrict__ pt, int32_t* __restrict__ seq_lens, int32_t* __restrict__ A,
    const T* __restrict__ k_new, const T* __restrict__ v_new, int32_t* __restrict__ counters) {
  constexpr int E = 16 / sizeof(T), LPV = D / E, VECTORS = kAppendThreads / LPV;
  constexpr int kBytes = mx4_block_bytes(PS, D), kPages = kMx4AppendTokens / PS + 1;
  __shared__ int s_phys[kPages];
  __shared__ int s_nok;
  const int b = blockIdx.x, tid = threadIdx.x, c = tid % LPV;
  const int pos0 = seq_lens[b];
  // (the score launch leaves them at zero, but a replayed step may find what another geometry's
  // call has left at their place)
  if (counters)
    for (int h = tid; h < g.hk; h += kAppendThreads)
      __hip_atomic_store(counters + ((int64_t)b * g.hk + h) * kSelCounterInts, 0, __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
  const int lp0 = pos0 >= 0 ? pos0 / PS : 0;
  const int npages = pos0 >= 0 ? (int)(((int64_t)pos0 + n_tok - 1) / PS) - lp0 + 1 : 0;
  if (tid == 0) s_nok = pos0 >= 0 ? n_tok : 0;
  __syncthreads();
  if (tid < npages) {
    const int lp = lp0 + tid, ph = lp < g.max_pages ? pt[(int64_t)b * g.max_pages + lp] : -1;
    const bool ok = ph >= 0 && ph < g.num_phys;
    s_phys[tid] = ok ? ph : -1;
    if (!ok) atomicMin(&s_nok, max(tid * PS - (pos0 - lp0 * PS), 0));
  }
  __syncthreads();
  const int n_ok = s_nok;
  if (n_ok <= 0) return;
  const int slot0 = pos0 - lp0 * PS;
  for (int x = tid / LPV; x < n_ok * g.hk; x += VECTORS) {
    const int j = x / g.hk, h = x - j * g.hk, at = slot0 + j;
    const int64_t src = ((int64_t)j * g.batch + b) * g.hk + h;  // [token][batch][h_k][d]
    const Codes<T> k(reinterpret_cast<const mx4_u32x4*>(k_new + src * D)[c]);
    const Codes<T> v(reinterpret_cast<const mx4_u32x4*>(v_new + src * D)[c]);
    const int64_t block = ((int64_t)s_phys[at / PS] * g.hk + h) * kBytes;
    k.template store_key<PS, D>(kc + block, at % PS, c);
    v.template store_value<PS, D>(vc + block, at % PS, c);
  }
  __syncthreads();  // keys are in the pages; every thread has read seq_lens[b]
  const int nlp = (slot0 + n_ok - 1) / PS + 1;
  for (int64_t x = tid; x < (int64_t)nlp * g.hk * D; x += kAppendThreads) {
    const int i = (int)(x % D), h = (int)(x / D % g.hk), page = (int)(x / D / g.hk);
    const char* block = kc + ((int64_t)s_phys[page] * g.hk + h) * kBytes;
    const int64_t row = ((int64_t)b * g.hk + h) * g.max_pages + lp0 + page;
    T* d = dg + row * 2 * D + i;
    const int first = page ? 0 : slot0, end = min(slot0 + n_ok - page * PS, PS);
    float lo = stored_key<PS, D>(block, first, i), hi = lo;
    if (first) {  // the page held keys before: its digest is widened
      lo = to_f32(d[0]);
      hi = to_f32(d[D]);
    }
    for (int t = first; t < end; ++t) {
      const float k = stored_key<PS, D>(block, t, i);
      if (k < lo) lo = k;
      if (hi < k) hi = k;
    }
    from_f32(lo, d);
    from_f32(hi, d + D);
    if (i == 0) A[row] = step - 1;  // Alg. 2's current-page rule
  }
  if (tid == 0) seq_lens[b] = pos0 + n_ok;
}

// The rows of one sequence's run of positions, a page of a KV head per workgroup, whose
// digest becomes that of all keys it then holds.  Prefill (n_upd 0): positions start .. end - 1 of
// sequence `seq`, whose length becomes `end`; UpdateKV: the n_upd last ones of every sequence.
constexpr int kRowsThreads = 128;

template <typename T, int PS, int D>
__global__ void __launch_bounds__(kRowsThreads) mx4_rows_kernel(
    Geometry g, int n_upd, int seq, int start, int end, char* kc, char* __restrict__ vc, T* __restrict__ dg,
    const int32_t* __restrict__ pt, int32_t* seq_lens, const T* __restrict__ k_src,
    const T* __restrict__ v_src) {
  constexpr int E = 16 / sizeof(T), LPV = D / E, NP = PS * LPV / kRowsThreads;
  constexpr int kBytes = mx4_block_bytes(PS, D);
  const int tid = threadIdx.x, c = tid % LPV, h = blockIdx.y;
  const int b = n_upd ? (int)blockIdx.z : seq;
  if (n_upd) end = seq_lens[b];
  const int from = n_upd ? max(end - n_upd, 0) : start;
  // the source's row of position 0
  const int64_t row0 = n_upd ? (int64_t)b * n_upd - ((int64_t)end - n_upd) : -(int64_t)start;
  const int lp = from / PS + blockIdx.x;
  if (!n_upd && blockIdx.x == 0 && h == 0 && tid == 0) seq_lens[seq] = end;
  if (lp >= g.max_pages || (int64_t)lp * PS >= end) return;
  const int phys = pt[(int64_t)b * g.max_pages + lp];
  if (phys < 0 || phys >= g.num_phys) return;
  const int64_t block = ((int64_t)phys * g.hk + h) * kBytes;
  const int s0 = max(from - lp * PS, 0), s1 = min(end - lp * PS, PS);
  mx4_u32x4 kr[NP], vr[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int t = tid / LPV + i * (kRowsThreads / LPV);
    if (t < s0 || t >= s1) continue;
    const int64_t src = (row0 + lp * PS + t) * g.hk + h;
    kr[i] = reinterpret_cast<const mx4_u32x4*>(k_src + src * D)[c];
    vr[i] = reinterpret_cast<const mx4_u32x4*>(v_src + src * D)[c];
  }
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int t = tid / LPV + i * (kRowsThreads / LPV);
    if (t < s0 || t >= s1) continue;
    Codes<T>(kr[i]).template store_key<PS, D>(kc + block, t, c);
    Codes<T>(vr[i]).template store_value<PS, D>(vc + block, t, c);
  }
  __syncthreads();
  T* d = dg + (((int64_t)b * g.hk + h) * g.max_pages + lp) * 2 * D;
  for (int i = tid; i < D; i += kRowsThreads) {
    float lo = stored_key<PS, D>(kc + block, 0, i), hi = lo;
    for (int t = 1; t < s1; ++t) {
      const float k = stored_key<PS, D>(kc + block, t, i);
      if (k < lo) lo = k;
      if (hi < k) hi = k;
    }
    from_f32(lo, d + i);
    from_f32(hi, d + D + i);
  }
}

// f(type, page size, head size) for the dims
template <typename F>
hipError_t with_shape(const Geometry& g, F f) {
  auto with_d = [&](auto t, auto ps) {
    return g.D == 128 ? f(t, ps, std::integral_constant<int, 128>{}) : f(t, ps, std::integral_constant<int, 64>{});
  };
  auto with_page = [&](auto t) {
    return g.P == 16 ? with_d(t, std::integral_constant<int, 16>{}) : with_d(t, std::integral_constant<int, 32>{});
  };
  return g.dtype == RETRO_BF16 ? with_page(bf16_t{}) : with_page(float{});
}

hipError_t launch_rows(const Geometry& g, const retro_kv_cache& c, dim3 grid, int n_upd, int seq, int start, int end,
                       const void* k, const void* v, hipStream_t s) {
  return with_shape(g, [&](auto t, auto ps, auto d) {
    using T = decltype(t);
    mx4_rows_kernel<T, decltype(ps)::value, decltype(d)::value><<<grid, kRowsThreads, 0, s>>>(
        g, n_upd, seq, start, end, (char*)c.k_cache, (char*)c.v_cache, (T*)c.digest, c.page_table, c.seq_lens,
        (const T*)k, (const T*)v);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_mx4_append_tokens(const Geometry& g, int step, const retro_kv_cache& c, int n_tok,
                                    const void* k_new, const void* v_new, hipStream_t s, int32_t* counters) {
  const size_t tok_elems = (size_t)g.batch * g.hk * g.D;
  return with_shape(g, [&](auto t, auto ps, auto d) {
    using T = decltype(t);
    for (int j0 = 0; j0 < n_tok; j0 += kMx4AppendTokens) {
      mx4_append_kernel<T, decltype(ps)::value, decltype(d)::value><<<g.batch, kAppendThreads, 0, s>>>(
          g, step, std::min(kMx4AppendTokens, n_tok - j0), (char*)c.k_cache, (char*)c.v_cache, (T*)c.digest,
          c.page_table, c.seq_lens, c.last_loaded, (const T*)k_new + j0 * tok_elems,
          (const T*)v_new + j0 * tok_elems, counters);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  });
}

hipError_t launch_mx4_prefill(const Geometry& g, const retro_kv_cache& c, int seq, int start, int n,
                              const void* k_src, const void* v_src, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  const int end = start + n;
  return launch_rows(g, c, dim3((unsigned)((end - 1) / g.P - start / g.P + 1), (unsigned)g.hk), 0, seq, start, end,
                     k_src, v_src, s);
}

hipError_t launch_mx4_update_kv(const Geometry& g, const retro_kv_cache& c, int n, const void* k_upd,
                                const void* v_upd, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  // the run [len - n, len) spans at most ceil(n / P) + 1 pages
  return launch_rows(g, c, dim3((unsigned)((n + g.P - 1) / g.P + 1), (unsigned)g.hk, (unsigned)g.batch), n, 0, 0, 0,
                     k_upd, v_upd, s);
}

}  // namespace retro
