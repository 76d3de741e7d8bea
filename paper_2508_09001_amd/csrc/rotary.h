// Ragged batches of rows (retro_chunk), per-head norms and rotations (retro_rotary):
// declarations shared by rotary.hip, chunk_attend.hip and the C ABI.
#pragma once

#include "internal.h"

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

}  // namespace retro
