// Ragged batches of rows (retro_chunk), per-head norms and rotations (retro_rotary):
// declarations shared by rotary.hip, chunk_attend.hip and the C ABI.
#pragma once

#include "roles.h"

namespace retro {

hipError_t launch_rotary_table(float* table, int positions, int rot_dim, double base, hipStream_t s);
bool rotate_qk_supported(const Geometry& g, int rows, bool q, bool k);
hipError_t launch_rotate_qk(const Geometry& g, const retro_rotary& r, const int32_t* positions,
                            int rows, const void* q, int64_t q_stride, const void* k,
                            int64_t k_stride, void* q_out, void* k_out, hipStream_t s);
bool append_rotary_supported(const Geometry& g, int n_rows);
hipError_t launch_append_rotary(const Geometry& g, int step, const retro_kv_cache& c,
                                const retro_chunk& ch, const retro_rotary& r, const void* q,
                                int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                int64_t v_stride, void* q_out, hipStream_t s);
// Rows of the cache as keys and values (kv_read.hip).
bool read_kv_supported(const Geometry& g, int n_rows);
hipError_t launch_read_kv(const Geometry& g, const retro_kv_cache& c, const retro_chunk& ch, void* k_out,
                          void* v_out, hipStream_t s);
// launch_chunk_attend over a cache in 4 bits (mx4_attend.hip), on the same workspace
hipError_t launch_mx4_attend(const Geometry& g, const retro_kv_cache& c, const retro_chunk& ch,
                             const void* q, int64_t q_stride, void* out, float* lse, void* workspace,
                             hipStream_t s);
bool chunk_attend_supported(const Geometry& g, int n_rows);
size_t chunk_workspace(const Geometry& g, int n_rows);
hipError_t launch_chunk_attend(const Geometry& g, const retro_kv_cache& c, const retro_chunk& ch,
                               const void* q, int64_t q_stride, void* out, float* lse,
                               void* workspace, hipStream_t s);

// Rows and first position of sequence b, cut to what the buffers hold; none for a
// sequence that takes no part.
struct Run {
  int row, n, pos;
};
__device__ __forceinline__ Run chunk_run(const retro_chunk& ch, int b) {
  Run r;
  r.row = ch.row_start[b];
  r.pos = ch.start_pos[b];
  const int end = min(ch.row_start[b + 1], ch.n_rows);
  // positions stay below 2^31
  r.n = r.row >= 0 && r.pos >= 0 ? min(max(end - r.row, 0), 0x7fffffff - r.pos) : 0;
  return r;
}

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
// Workgroups for every sequence's pages, at most n / P + 2 of each, in eights (an XCD's
// workgroups are every eighth), `kinds` for a page.
inline int64_t page_blocks(const Geometry& g, int n_rows, int kinds) {
  const int64_t pages = n_rows / g.P + 2 * (int64_t)std::min(g.batch, n_rows);
  return (pages + 7) / 8 * 8 * kinds;
}

}  // namespace retro
