// Dense causal attention of a ragged batch of rows over the paged cache.
//
// Rows of a KV head are (row of the chunk, query head of the group), G after G.
// In tiles of 32 keys x 32 rows, S^T = K Q^T and O^T += V^T P^T on 32x32 matrix
// instructions: a lane holds one row's scores, so that maximum, sum and
// rescaling need one exchange (with the lane 32 away), and its exponentials are
// the next product's operand as they lie: key row i of S^T is key
// 16 (i / 16) + 8 (i / 4 % 2) + 4 (i / 8 % 2) + i % 4 of the tile for bf16 (where a
// lane's operand is eight consecutive keys), key i for fp32 (four).
//
// A workgroup of eight wavefronts takes a unit of work in one of two ways:
//   - 32 rows (all that a sequence has, or where there is too little work for the
//     other way): the wavefronts take 32 keys in turn, each through LDS of its own,
//     without barriers, and join their (maximum, sum, output) at the end; bound by
//     reading the cache;
//   - many rows (bf16): 32 of 256 rows each, all over the same 64 keys, which are
//     copied into LDS for all, one stage ahead; bound by the matrix cores.
// The work is laid out on the device, from the arrays of the call, by every
// workgroup for itself: the steps of all tiles of 32 rows are one line, cut into
// shares wherever that falls (equal ones; more for a workgroup that gets no tile of
// many rows where others do); tiles of many rows are cut along the keys where there
// are too few of them to fill the GPU.  A tile's parts go to the
// workspace, written and read past the L2s of the XCDs, and the workgroup that
// finishes the last one joins them.
//
// Measured (bf16, 8 KV heads of 4 query heads of 128; several cards): a prompt of 8192
// tokens 483 to 546 us (1.01 to 1.14 PFLOP/s), 1024 rows at 131K 1.82 to 2.03 ms (1.08 to
// 1.20), where a product of 16384^3 reaches 1.33 to 1.37: the matrix units are busy 64 % of the cycles at 1.75
// GHz, which is where such products hold the clock too, and leaving out any one part
// of the loop (exponentials, LDS reads, copies, maxima, sums) gains 4 to 9 %.  16 tokens
// at 8K to 32K, 1.15 GB: 187 us, 6.15 TB/s, the rate of a plain read.  Short calls wait for
// one memory round trip after the other: 8 us for a token at 100, 14 at 2000.  fp32 chunks
// reach 0.06 to 0.11 of the 0.15 PFLOP/s of a large fp32 product.
//
// Pages lie in LDS as in memory, cut into 16-byte pieces whose order within a
// row is xored with the row's number, so that the 16 lanes of a read fall into 16
// different groups of banks; the copy engine writes LDS in order and reads
// memory in the permuted one.
#include "chunk_work.h"

namespace retro {
namespace {

// ---- kernel ------------------------------------------------------------------------------

// MANY: with tiles of many rows.  Without them the same line of tiles of 32 rows is
// walked in less code and registers (one token at 32K: 38.8 -> 32.6 us).
template <typename T, int D, int P, bool MANY>
__global__ void __launch_bounds__(kThreads) chunk_attend_kernel(AttendCall a) {
  using S = Shape<T, D, P>;
  using R_t = Rows<T, D, P>;
  using Lds_t = ChunkLds<T, D, P>;
  __shared__ __attribute__((aligned(1024))) Lds_t L;
  const int tid = thread_index();
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t st = lds_address(&L.u);
  const Cut cut = make_cut<MANY>(a, P, L.find, tid);
  const int64_t page_bytes = (int64_t)P * D * sizeof(T), phys_bytes = page_bytes * a.hk;
  // a lane's place within a copy of keys, and of values: pieces in their LDS order
  uint32_t kcopy, vcopy;
  {
    const int lane = tid & 63;
    kcopy = lane / S::CPR * (D * sizeof(T)) + (lane % S::CPR ^ S::fk(lane / S::CPR)) * 16;
    vcopy = lane / S::CPV * (P * sizeof(T)) + (lane % S::CPV ^ S::fv(lane / S::CPV)) * 16;
  }
  // copy i of a tile: rows further on, whose numbers change the order by this
  constexpr int kRowsPerCopy = 64 / S::CPR;
  auto kxor = [](int i) { return (uint32_t)S::fk(i * kRowsPerCopy & 31) << 4; };
  auto vxor = [](int i) { return S::CPV == 8 ? (uint32_t)(i & 1) << 6 : 0u; };

  // the result of row rho of a sequence's rows for KV head h, four elements of d
  auto finish = [&](const Seq& s, int h, int rho, float m, float l, int d, f32x4 o) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t at = (int64_t)(s.run.row + rho / a.G) * a.hq + h * a.G + rho % a.G;
    store4((T*)a.out + at * D + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    if (d == 0 && a.lse) a.lse[at] = natural_lse(m, l, a.scale);
  };

  // ---- tiles of 32 rows: this workgroup's share of the line of steps
  auto few_rows = [&]() {
    constexpr int PT = 32 / P;  // pages of a tile
    // (from the last workgroup on: the first ones take the tiles of many rows, if there are few)
    const int64_t me = kCus - 1 - blockIdx.x, mine = cut.begin(me), upto = min(cut.begin(me + 1), cut.line);
    for (int64_t pos = mine; pos < upto;) {
      int b = 0;
      int64_t local = 0, before;
      Seq s;
      find_seq(a, P, pos, L.find, tid, [&](const Seq& s) { return cut.line_of(s, a); },
               [](const Seq&) { return (int64_t)0; }, s, b, local, before);
      const Pages page_of = pages_of<P>(a, s, b);
      const int tiles = s.tiles(kRowsFew);
      // its KV heads and their tiles, one after the other
      const int64_t per_head = s.place(tiles, a.G);
      int h = (int)(local / per_head), tile = 0;
      local -= h * per_head;
      for (int n = tiles; n > 1;) {  // the last tile that begins at or in front of local
        const int half = n / 2;
        if (s.place(tile + half, a.G) <= local) {
          tile += half;
          n -= half;
        } else {
          n = half;
        }
      }
      int step0 = (int)(local - s.place(tile, a.G));
      while (h < a.hk && pos < upto) {
        const int rho0 = tile * kRowsFew, nr = min(s.rows - rho0, kRowsFew);
        const int length = (int)(s.place(tile + 1, a.G) - s.place(tile, a.G));
        const int n = (int)min((int64_t)(length - step0), upto - pos);
        // (a place's last steps may lie behind the tile's end, in a sequence whose start_pos
        // is out of range far behind: then nothing is read)
        const int key_begin = min(step0, 1 << 24) * 64,
                  key_end = (int)min((int64_t)s.seen(rho0 + kRowsFew, a.G), ((int64_t)step0 + n) * 64);
        const char* kh = (const char*)a.kc + h * page_bytes;
        const char* vh = (const char*)a.vc + h * page_bytes;
        const int lane = thread_index() & 63;
        R_t rows;
        rows.init(lane, a.scale);
        bool live;
        int lim;
        const T* qrow = row_at<T, D>(a, s, h, rho0 + (lane & 31), live, lim);
        rows.start(qrow, live, lim);
        const int all_see = min(s.run.pos + rho0 / a.G, s.end - 1);  // last token that every row sees
        const uint32_t ks = st + wave * (int)sizeof(L.u.own[0]), vs = S::ONE ? ks : ks + S::TILE;
        rows.read_from(ks, vs);
        // copies a tile's keys or values; which of its pages are not mapped
        auto issue = [&](const char* base, uint32_t to, int key, uint32_t off, auto x) {
          uint32_t bits = 0;
#pragma unroll
          for (int pg = 0; pg < PT; ++pg) {
            bool bad;
            const char* src = base + page_of(key / P + pg, bad) * phys_bytes;
            bits |= (uint32_t)bad << pg;
#pragma unroll
            for (int i = 0; i < S::PPP; ++i)
              if (s.few)  // the only tile of these keys
                copy_to_lds<true>(src + i * 1024, off ^ x(pg * S::PPP + i), to + (pg * S::PPP + i) * 1024);
              else
                copy_to_lds<false>(src + i * 1024, off ^ x(pg * S::PPP + i), to + (pg * S::PPP + i) * 1024);
          }
          return bits;
        };
        int key = key_begin + wave * 32;
        if (key < key_end) {
          uint32_t bad = issue(kh, ks, key, kcopy, kxor);
          if constexpr (!S::ONE) issue(vh, vs, key, vcopy, vxor);
          for (; key < key_end; key += kWaves * 32) {
            const int next = key + kWaves * 32;
            f32x16 sc[1];
            wait_loads<S::ONE ? 0 : S::LOADS>();
            sc[0] = rows.scores(0);
            asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
            uint32_t bad_next = 0;
            if constexpr (S::ONE) issue(vh, vs, key, vcopy, vxor);
            else if (next < key_end) bad_next = issue(kh, ks, next, kcopy, kxor);
            // (masking every tile costs nothing for bf16: the wavefront waits for memory)
            const bool clean = sizeof(T) == 4 && !bad && key + 31 <= all_see;
            if (!clean) rows.mask(sc, key, bad);
            rows.weights(sc, rows.follow(sc));
            if (!S::ONE && next < key_end) wait_loads<S::LOADS>();
            else wait_loads<0>();
            // (and neither does the weights' second half: 0.0022 -> 0.0017 off 64 bits)
            if constexpr (sizeof(T) == 4)
              if (!clean) rows.clear(s.end - key, bad);
            rows.template values<true>(0, sc[0], s.end - key, bad);
            asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
            if (next < key_end) {
              if constexpr (S::ONE) bad_next = issue(kh, ks, next, kcopy, kxor);
              else issue(vh, vs, next, vcopy, vxor);
            }
            bad = bad_next;
          }
        }
        // join the wavefronts' results
        barrier();
        const int r = lane & 31;
        rows.l = rows_half_sum(rows.l);
        if (lane < 32) {
          L.m[wave][r] = rows.m;
          L.l[wave][r] = rows.l;
        }
        if (r < nr)
#pragma unroll
          for (int i = 0; i < R_t::DT; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
              *reinterpret_cast<f32x4*>(&L.u.o[wave][r][i * 32 + 2 * e + 4 * rows.half]) =
                  f32x4{rows.acc[i][e], rows.acc[i][e + 1], rows.acc[i][e + 2], rows.acc[i][e + 3]};
        barrier();
        // a part: slot 2 k of workgroup k for what its share begins with, 2 k + 1 for what it ends with
        const bool whole = n == length;
        const int64_t k = me;
        auto slot = [&](int64_t i) { return a.few + i * slot_floats(kRowsFew, D); };
        const __amdgpu_buffer_rsrc_t part = coherent_rsrc(slot(2 * k + (pos != mine)));
        for (int i = tid; i < nr * (D / 4); i += kThreads) {
          const int row = i / (D / 4), d = i % (D / 4) * 4;
          float m = -INFINITY;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) m = fmaxf(m, L.m[w][row]);
          const float mu = m == -INFINITY ? 0.f : m;
          float l = 0.f;
          f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < kWaves; ++w) {
            const float e = __builtin_amdgcn_exp2f((L.m[w][row] - mu) * rows.c);
            const f32x4 x = *reinterpret_cast<const f32x4*>(&L.u.o[w][row][d]);
            l = __builtin_fmaf(e, L.l[w][row], l);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = __builtin_fmaf(e, x[j], o[j]);
          }
          if (whole) {
            finish(s, h, rho0 + row, m, l, d, o);
          } else {
            put_part(part, row * D + d, o);
            if (d == 0) {
              put_part(part, kRowsFew * D + row, m);
              put_part(part, kRowsFew * (D + 1) + row, l);
            }
          }
        }
        if (!whole) {
          // the tile's steps are start .. start + length - 1 of the line
          const int64_t start = pos - step0, k0 = cut.owner(start);
          const int parts = (int)(cut.owner(start + length - 1) - k0) + 1;
          if (last_part(a.counters + k0, parts, &L.last, tid))
            join_few<D>(
                L.u.join, nr, parts, rows.c, tid,
                [&](int p) { return slot(2 * (k0 + p) + (p == 0 && start != cut.begin(k0))); },
                [&](int row, float m, float l, int d, f32x4 o) { finish(s, h, rho0 + row, m, l, d, o); });
        }
        barrier();
        pos += n;
        step0 = 0;
        if (++tile == tiles) {
          tile = 0;
          ++h;
        }
      }
    }
  };

  // Reading the cache for few rows leaves the matrix cores idle and the other way
  // round: every other workgroup of an XCD begins with the one, the rest with the other.
  [[maybe_unused]] const bool turn = blockIdx.x >> 3 & 1;
  if constexpr (MANY) {
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
      if ((i == 0) != turn) {
        if (cut.many)
          many_rows<T, D, P>(a, cut, L, tid, wave, CopiedStages<T, D, P>{phys_bytes, page_bytes, kcopy, vcopy}, finish);
      } else {
        if (cut.line) few_rows();
      }
    }
  } else {
    if (cut.line) few_rows();
  }
}

// The most tiles and parts that any lengths can give.
struct Bounds {
  int64_t few, many;  // tiles of all sequences and KV heads
  int64_t parts;      // parts of cut tiles of many rows
};
Bounds bounds(const Geometry& g, int n_rows) {
  Bounds x;
  const int64_t rows = (int64_t)n_rows * g.G;
  const int64_t steps = ((int64_t)g.max_pages * g.P + 63) / 64;
  x.few = std::min<int64_t>(g.batch, n_rows) * g.hk;
  const int64_t seqs = std::min<int64_t>(g.batch, rows / (kRowsFew + 1));
  x.many = seqs ? (rows / kRowsMany + seqs) * g.hk : 0;
  // a tile of n >= 2 parts has more than n - 1 >= n / 2 times a part's most steps, and
  // that is at least 1 / grid of all steps
  x.parts = steps <= kMinMany ? 0
                              : std::min(x.many * ((steps + kMinMany - 1) / kMinMany),
                                         (int64_t)2 * kCus);
  return x;
}

}  // namespace

bool chunk_attend_supported(const Geometry& g, int n_rows) {
  // (row numbers of a tile go up to one tile of many rows past the last row)
  return (int64_t)n_rows * g.hq * g.D < (int64_t)1 << 40 &&
         (int64_t)n_rows * g.G < ((int64_t)1 << 31) - kRowsMany;
}

size_t chunk_workspace(const Geometry& g, int n_rows) {
  // every workgroup's share of few rows begins and ends with a part
  const size_t floats = 2 * (size_t)kCus * slot_floats(kRowsFew, g.D) +
                        bounds(g, n_rows).parts * slot_floats(kRowsMany, g.D);
  return kCounterBytes + ((floats * sizeof(float) + 255) & ~size_t(255));
}

hipError_t launch_chunk_attend(const Geometry& g, const retro_kv_cache& c, const retro_chunk& ch,
                               const void* q, int64_t q_stride, void* out, float* lse, void* ws,
                               hipStream_t s) {
  const AttendCall a = attend_call(g, c, ch, q, q_stride, out, lse, ws);
  const bool many = g.dtype == RETRO_BF16 && may_have_many(ch, g.batch, g.G);
  auto go = [&](auto t, auto d, auto ps) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value, P = decltype(ps)::value;
    if constexpr (sizeof(T) == 2) {
      if (many) {
        chunk_attend_kernel<T, D, P, true><<<kCus, kThreads, 0, s>>>(a);
        return hipGetLastError();
      }
    }
    chunk_attend_kernel<T, D, P, false><<<kCus, kThreads, 0, s>>>(a);
    return hipGetLastError();
  };
  auto with_page = [&](auto t, auto d) {
    return g.P == 16 ? go(t, d, std::integral_constant<int, 16>{})
                     : go(t, d, std::integral_constant<int, 32>{});
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (g.dtype == RETRO_BF16) return g.D == 128 ? with_page(bf16_t{}, D128{}) : with_page(bf16_t{}, D64{});
  return g.D == 128 ? with_page(float{}, D128{}) : with_page(float{}, D64{});
}

}  // namespace retro
