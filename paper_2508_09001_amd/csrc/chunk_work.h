// How attention over the paged cache by a ragged batch of rows is laid out over the
// GPU, and what a wavefront does with tiles of 32 keys and 32 rows: shared by
// chunk_attend.hip (pages in the rows' type) and mx4_attend.hip (pages in 4 bits).
#pragma once

#include "roles.h"
#include "rotary.h"

namespace retro {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kRowsFew = 32;             // rows of a unit in the first way
constexpr int kRowsMany = 32 * kWaves;   // and in the second
constexpr int kCus = 256;
constexpr int kMinMany = 8, kMinFew = 4; // least steps of 64 keys of a part
// What a step of a tile costs a workgroup while others do the other kind: 0.8 and 2.1 us
// alone, each longer beside the other (us with 2 to 5, 1 to 2 and 3 to 5: a chunk of 100
// rows beside 15 tokens at 4K to 16K 153, 148, 139; of 256 beside 32 at 2K to 8K 145, 145,
// 166; of 1024 beside 63 at 0.5K to 2K 126, 134, 113)
constexpr int64_t kFewCost = 1, kManyCost = 2;
constexpr int kScans = 6;                // prefix sums made together

struct AttendCall {
  retro_chunk ch;
  const void *kc, *vc;
  const int32_t *pt, *seq_lens;
  const void* q;
  int64_t q_stride;
  void* out;
  float* lse;
  int32_t* counters;
  float *few, *many;  // parts' results
  int batch, hk, G, hq, max_pages, num_phys;
  float scale;
};

// ---- the work of a call ----------------------------------------------------------------

struct Seq {
  Run run;
  int end;    // stored tokens that the rows may see
  int rows;   // of a KV head
  bool few;   // they fit one tile of 32
  __device__ __forceinline__ int tiles(int of) const { return (int)(((int64_t)rows + of - 1) / of); }
  __device__ __forceinline__ int steps() const { return max((end + 63) / 64, 1); }  // of 64 keys
  // tokens that the rows in front of `upto` see at most
  __device__ __forceinline__ int seen(int upto, int G) const {
    return min(end, run.pos + (min(upto, rows) - 1) / G + 1);
  }
  // Where tile i of 32 rows begins in the line of steps of a KV head's tiles.  A tile's
  // place is as long as its steps or a little longer: tile j sees pos + (32 (j + 1) - 1) / G
  // + 1 tokens, of which the sum over j < i has no simple form, but a bound on it has.
  __device__ __forceinline__ int64_t place(int64_t i, int G) const {
    if (few) return i * steps();
    return (i * ((int64_t)run.pos + 1) * G + 16 * i * (i + 1)) / (64 * (int64_t)G) + 2 * i;
  }
};

__device__ __forceinline__ Seq make_seq(Run run, int end, int G) {
  const int rows = run.n * G;
  return Seq{run, end, rows, rows <= kRowsFew};
}
__device__ __forceinline__ Seq load_seq(const AttendCall& a, int P, int b) {
  Seq s = make_seq(b < a.batch ? chunk_run(a.ch, b) : Run{0, 0, 0}, 0, a.G);
  const int len = b < a.batch ? a.seq_lens[b] : 0;
  s.end = (int)min((int64_t)min(max(len, 0), s.run.pos + s.run.n), (int64_t)a.max_pages * P);
  return s;
}

// What every workgroup agrees on.
struct Cut {
  bool all_line;      // no tiles of many rows
  int64_t line;       // steps of all tiles of 32 rows, of all KV heads
  int64_t share;      // a workgroup's share of them
  int64_t first, long_share;  // the first ones', that have no tile of many rows
  int64_t many;       // steps of all tiles of many rows
  int part;           // most steps of a part of such a tile
  __device__ __forceinline__ bool on_line(const Seq& s) const { return s.few || all_line; }
  // where workgroup k's share of the line begins, and whose share a step is in
  __device__ __forceinline__ int64_t begin(int64_t k) const {
    return min(k, first) * long_share + max(k - first, (int64_t)0) * share;
  }
  __device__ __forceinline__ int64_t owner(int64_t step) const {
    const int64_t past = step - first * long_share;
    return past < 0 ? step / long_share : first + past / share;
  }
  __device__ __forceinline__ int64_t line_of(const Seq& s, const AttendCall& a) const {
    return on_line(s) ? a.hk * s.place(s.tiles(kRowsFew), a.G) : 0;
  }
};

// A prefix sum over a wavefront, as wave_inclusive_scan, in 64 bits.
template <int CTRL, int ROW_MASK, bool BOUND_ZERO>
__device__ __forceinline__ int64_t dpp_i64(int64_t x) {
  const uint32_t lo = dpp_i<CTRL, ROW_MASK, BOUND_ZERO>((int)(uint32_t)x);
  const uint32_t hi = dpp_i<CTRL, ROW_MASK, BOUND_ZERO>((int)(x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int64_t wave_scan_i64(int64_t x) {
  x += dpp_i64<0x111, 0xF, true>(x);
  x += dpp_i64<0x112, 0xF, true>(x);
  x += dpp_i64<0x114, 0xF, true>(x);
  x += dpp_i64<0x118, 0xF, true>(x);
  x += dpp_i64<0x142, 0xA, false>(x);
  x += dpp_i64<0x143, 0xC, false>(x);
  return x;
}
__device__ __forceinline__ int64_t read_lane(int64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)x, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(x >> 32), lane);
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int64_t last_lane(int64_t x) { return read_lane(x, 63); }
// Prefix sums of N values over the workgroup's threads, and their totals.
template <int N>
struct Scan {
  int64_t of[N], total[N];
};
template <int N>
__device__ __forceinline__ void block_scan(Scan<N>& s, int64_t (&scratch)[kScans][kWaves], int tid) {
#pragma unroll
  for (int j = 0; j < N; ++j) {
    s.of[j] = wave_scan_i64(s.of[j]);
    if ((tid & 63) == 63) scratch[j][tid >> 6] = s.of[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < N; ++j) {
    int64_t base = 0;
    s.total[j] = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      if (i < tid >> 6) base += scratch[j][i];
      s.total[j] += scratch[j][i];
    }
    s.of[j] += base;
  }
  __syncthreads();
}

// Up to 64 sequences every wavefront does by itself, a lane for each: no barrier, and
// little code (a workgroup that runs once waits for much of it to be fetched).
struct FindLds {
  int64_t scratch[kScans][kWaves];
  int64_t local, before;
  int4 first[kThreads];  // run and end of the first sequences
  int b;
};
__device__ __forceinline__ Seq first_seq(const FindLds& L, int b, int G) {
  const int4 x = L.first[b];
  return make_seq(Run{x.x, x.y, x.z}, x.w, G);
}

// Tiles of 256 rows read a key once from the L2 where those of 32 read it eight times,
// but a part of one is long (eight steps, or all) and its joining moves 256 rows.  So
// where there are few of them, with long sequences and little work in all, all tiles
// are of 32 rows (us, 32 against 256 rows; 8 KV heads of 4 query heads): 64 rows at 2000
// tokens 34 and 47, 128 at 4000 49 and 57; but 256 at 2000 53 and 50, 512 at 4000 136
// and 69, 128 rows of a new prompt 33 and 21.  fp32 tiles always are of 32 rows: its
// matrix instructions are 16 times slower, and the reading does not show.
//
// MX4: over a cache in 4 bits a step of 32 rows costs a workgroup 0.42 us, a tile besides 20
// where a workgroup has several, a part 0.4; one of 256 rows 2.0, and where tiles are cut
// 8 and 1.6 a part (8 KV heads of 4 query heads, us with 32 and 256 rows: 64 rows at 8000 35
// and 68, at 32000 74 and 116; 128 at 8000 48 and 73, at 32000 125 and 117; 256 at 2000 40 and
// 50, at 8000 77 and 75; 512 at 2000 61 and 55; 1000 at 8000 260 and 160; a chunk of 100 beside 15
// tokens at 2K to 8K 60 and 79).  Uncut tiles of 256 rows need no such question: 128 rows of a new
// prompt 27 and 21.
template <bool MANY, bool MX4 = false>
__device__ __forceinline__ Cut make_cut(const AttendCall& a, int P, FindLds& L, int tid) {
  constexpr int64_t kManyCost = MX4 ? 5 : retro::kManyCost;
  enum { kLine, kLineTiles, kSmall, kSmallTiles, kMany, kTiles, kSums };
  static_assert(kSums <= kScans, "sums made together");
  Scan<kSums> x;
  for (int j = 0; j < kSums; ++j) x.of[j] = 0;
  const bool wavefront = a.batch <= 64;
  for (int b = wavefront ? tid & 63 : tid; b < a.batch; b += kThreads) {
    const Seq s = load_seq(a, P, b);
    if (b < kThreads) L.first[b] = int4{s.run.row, s.run.n, s.run.pos, s.end};  // (the same from every wavefront)
    const int small = s.tiles(kRowsFew);
    const int64_t line = a.hk * s.place(small, a.G);
    if (!MANY || s.few) {
      x.of[kLine] += line;
      x.of[kLineTiles] += (int64_t)a.hk * small;
    } else {
      const int64_t tiles = (int64_t)a.hk * s.tiles(kRowsMany);
      x.of[kSmall] += line;
      x.of[kSmallTiles] += (int64_t)a.hk * small;
      x.of[kMany] += tiles * s.steps();
      x.of[kTiles] += tiles;
    }
  }
  if (wavefront) {
#pragma unroll
    for (int j = 0; j < kSums; ++j) x.total[j] = last_lane(wave_scan_i64(x.of[j]));
    __syncthreads();
  } else {
    block_scan(x, L.scratch, tid);
  }
  const int64_t n = gridDim.x, many = x.total[kMany], tiles = x.total[kTiles];
  Cut c;
  c.all_line = !MANY || (many < 5 * n && 8 * tiles < n && many > 16 * tiles);
  if constexpr (MANY && MX4) {
    // (in microseconds; no quotients of 64-bit integers, which took 3 of them)
    auto over = [](float a, float b) { return a * __builtin_amdgcn_rcpf(b); };
    const float cus = (float)n, of_many = (float)tiles, of_few = (float)x.total[kSmallTiles];
    const float steps = over((float)many, fmaxf(of_many, 1.f));
    const float whole = of_many < cus ? over(steps, floorf(over(cus, fmaxf(of_many, 1.f)))) : 0.f;
    const float part = fmaxf(fmaxf(over((float)many, cus), whole), (float)kMinMany);
    const float as_many = 2.0f * part + 10.f + 1.6f * over(steps, part);
    const float as_few = 0.42f * over((float)x.total[kSmall], cus) +
                         (of_few > cus ? 20.f * (over(of_few, cus) - 1.f) : 0.4f * over(cus, fmaxf(of_few, 1.f)));
    c.all_line = steps > part && as_few < as_many;
  }
  c.line = x.total[kLine] + (c.all_line ? x.total[kSmall] : 0);
  c.many = c.all_line ? 0 : many;
  // (tiles shorter than four steps are a share each: one after the other they would take
  // as many round trips: 33 sequences of 33 tokens 22 us, 13 so)
  const int64_t of_line = x.total[kLineTiles] + (c.all_line ? x.total[kSmallTiles] : 0);
  int64_t least = MX4 ? 1 : of_line ? min((c.line + of_line - 1) / of_line, (int64_t)kMinFew) : 1;
  if constexpr (MX4) {
    // A tile of up to eight steps is not cut, a longer one into some 32 parts at most, whose
    // joining costs as much as the reading of as many codes does (a token at 500 tokens 13.4 ->
    // 10.4 us, at 32000 of 2 KV heads of 16 query heads in 128, 64, 32 and 16 parts 45, 31, 26 and
    // 28).
    const int64_t steps = c.line > 8 * of_line ? (int64_t)((float)c.line * __builtin_amdgcn_rcpf((float)of_line)) : 1;
    least = c.line > 8 * of_line ? max((int64_t)kMinFew, (steps + 31) / 32)
                                 : of_line ? (c.line + of_line - 1) / of_line : 1;
  }
  c.share = max((c.line + n - 1) / n, least);
  c.first = c.long_share = 0;
  // A part's most steps: all workgroups' share of the work, but no less than that gives
  // every workgroup one part where there are fewer tiles than workgroups (of tiles of
  // unlike lengths every other one has a part more; of like ones all have as many): a
  // second round of some costs as much as one of all.  1332 rows of 8 KV heads and two
  // sequences at 420 tokens 82 -> 52 us.
  int64_t part = (kManyCost * c.many + kFewCost * c.line + kManyCost * n - 1) / (kManyCost * n);
  if (MANY && c.many && tiles <= n) {
    const int64_t work = part;
    part = max(part, (c.many + n - tiles / 2 - 1) / (n - tiles / 2));
    const int64_t steps = (c.many + tiles - 1) / tiles;
    if ((steps + part - 1) / part * tiles > n) part = (steps + n / tiles - 1) / (n / tiles);
    part = max(part, (int64_t)kMinMany);
    if (c.line) {
      // The workgroups without a part take as much more of the line, so that some read
      // while others multiply (us, against equal shares of the line: a chunk of 256 rows
      // beside 32 tokens at 2K to 8K 215 -> 145, of 100 beside 15 at 4K to 16K 253 -> 148).
      Scan<1> y;
      y.of[0] = 0;
      for (int b = wavefront ? tid & 63 : tid; b < a.batch; b += kThreads) {
        const Seq s = b < kThreads ? first_seq(L, b, a.G) : load_seq(a, P, b);
        if (!s.few) y.of[0] += (int64_t)a.hk * s.tiles(kRowsMany) * ((s.steps() + part - 1) / part);
      }
      if (wavefront) y.total[0] = last_lane(wave_scan_i64(y.of[0]));
      else block_scan(y, L.scratch, tid);
      c.first = max(n - y.total[0], (int64_t)0);
      if (c.first) {
        c.long_share = max(min((kManyCost * work + kFewCost - 1) / kFewCost, (c.line + c.first - 1) / c.first), least);
        const int64_t left = max(c.line - c.first * c.long_share, (int64_t)0);
        c.share = max((left + n - c.first - 1) / max(n - c.first, (int64_t)1), least);
      }
    }
  }
  c.part = (int)min(max(part, (int64_t)kMinMany), (int64_t)1 << 30);
  return c;
}

// The sequence b that item u belongs to, where a sequence has count(seq) items, and
// the item's number within it; before: the sum of other(seq) over the sequences in front.
template <typename Count, typename Other>
__device__ __forceinline__ bool find_seq(const AttendCall& a, int P, int64_t u, FindLds& L, int tid,
                                         Count&& count, Other&& other, Seq& seq, int& b, int64_t& local,
                                         int64_t& before) {
  if (a.batch <= 64) {
    const int lane = tid & 63;
    const Seq s = first_seq(L, min(lane, a.batch - 1), a.G);
    const int64_t n = lane < a.batch ? count(s) : 0, f = lane < a.batch ? other(s) : 0;
    const int64_t upto = wave_scan_i64(n);
    const uint64_t past = wave_ballot(upto > u);
    if (!past) return false;
    b = __builtin_ctzll(past);
    local = u - (read_lane(upto, b) - read_lane(n, b));
    before = read_lane(wave_scan_i64(f) - f, b);
    auto of_b = [&](int v) { return __builtin_amdgcn_readlane(v, b); };
    seq = make_seq(Run{of_b(s.run.row), of_b(s.run.n), of_b(s.run.pos)}, of_b(s.end), a.G);
    return true;
  }
  int64_t base = 0, obase = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
    const Seq s = b0 ? load_seq(a, P, b0 + tid)
                     : first_seq(L, min(tid, a.batch - 1), a.G);
    const bool is = b0 + tid < a.batch;
    const int64_t n = is ? count(s) : 0, f = is ? other(s) : 0;
    Scan<2> x{{n, f}, {}};
    block_scan(x, L.scratch, tid);
    const int64_t upto = base + x.of[0];
    if (u >= upto - n && u < upto) {
      L.b = b0 + tid;
      L.local = u - (upto - n);
      L.before = obase + x.of[1] - f;
    }
    __syncthreads();
    if (u < base + x.total[0]) {
      auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
      b = uniform(L.b);
      if (b < kThreads) {
        const int4 x = L.first[b];
        seq = make_seq(Run{uniform(x.x), uniform(x.y), uniform(x.z)}, uniform(x.w), a.G);
      } else {
        seq = load_seq(a, P, b);
      }
      local = L.local;
      before = L.before;
      __syncthreads();
      return true;
    }
    base += x.total[0];
    obase += x.total[1];
  }
  return false;
}

// A part's result in the workspace: outputs not yet divided, maxima, sums.
constexpr int slot_floats(int rows, int D) { return rows * (D + 2); }
constexpr int kCounters = 2 * kCus + kCus;  // parts done of each cut tile; zero between calls
constexpr size_t kCounterBytes = (kCounters * sizeof(int32_t) + 255) & ~size_t(255);

// A call's arguments on a workspace as chunk_workspace sizes it.
inline AttendCall attend_call(const Geometry& g, const retro_kv_cache& c, const retro_chunk& ch, const void* q,
                              int64_t q_stride, void* out, float* lse, void* ws) {
  float* few = reinterpret_cast<float*>((char*)ws + kCounterBytes);
  return AttendCall{ch,
                    c.k_cache,
                    c.v_cache,
                    c.page_table,
                    c.seq_lens,
                    q,
                    q_stride,
                    out,
                    lse,
                    (int32_t*)ws,
                    few,
                    few + 2 * (size_t)kCus * slot_floats(kRowsFew, g.D),
                    g.batch,
                    g.hk,
                    g.G,
                    g.hq,
                    g.max_pages,
                    g.num_phys,
                    g.sm_scale};
}

// Whether the call gets the kernel that also takes tiles of many rows, which costs a
// call without them 3 us and 5 to 18 % (a token each of 33 to 512 sequences at 60 to 8000
// tokens).  The device knows the lengths; the host may know the longest one: up to 32 rows
// there are no such tiles, and above 128 they are worth having (a chunk beside empty ranges,
// us without and with them: 280 rows of 256 sequences at 4000 96 and 57, 540 of 512 at 4000
// 146 and 69, at 0 52 and 31; 64 of 64 at 4000 34 and 37).  In between, and where it is
// unknown, every sequence is taken to have a row, which bounds the longest.
inline bool may_have_many(const retro_chunk& ch, int batch, int G) {
  const int64_t longest = (int64_t)std::min(ch.longest, ch.n_rows) * G;
  if (longest > 4 * kRowsFew) return true;
  return ((int64_t)ch.n_rows - batch + 1) * G > 4 * kRowsFew && (longest <= 0 || longest > kRowsFew);
}

// ---- LDS pieces ----------------------------------------------------------------------

template <typename T, int D, int P>
struct Shape {
  static constexpr int E = 16 / sizeof(T);       // elements of a piece
  static constexpr int KB = 32;                  // keys of a tile
  static constexpr int CPR = D / E;              // pieces of a key row
  static constexpr int CPV = P / E;              // pieces of a value row (one element of d of a page)
  static constexpr int TILE = KB * D * sizeof(T);  // bytes of a tile's keys (and of its values)
  static constexpr int KEYS = 64;                // keys of a shared stage
  static constexpr int NB = KEYS / KB;
  static constexpr int STAGE = 2 * NB * TILE;    // bytes of a stage: keys, then values
  static constexpr int LOADS = TILE / 1024;      // wavefront copies of a tile's keys (or values)
  static constexpr int PPP = P * D * (int)sizeof(T) / 1024;  // copies of a page
  // In the first way a wavefront has one buffer for a tile's keys and one for its values,
  // or where that is too much LDS (fp32 of d 128) one for both in turn, the other
  // wavefront of the SIMD multiplying meanwhile (us, against two for half as many
  // wavefronts: 1024 rows at 1024 328 -> 266, a token at 32K 80 -> 64).
  static constexpr bool ONE = TILE > 8192;
  static constexpr int OROW = D + 4;             // row of the joining buffer
  static constexpr int QC = CPR / 2;             // pieces of a row per lane half
  // order of a key row's pieces, and of a value row's
  static __device__ __forceinline__ int fk(int row) { return CPR == 8 ? (row >> 1) & 7 : row & 15; }
  static __device__ __forceinline__ int fv(int d) { return d / (16 / CPV) % CPV; }
};

// Joining parts.  32 rows: weights of some parts, what rows have so far, and several
// groups of lanes' sums.
constexpr int kJoinFew = 64;
struct JoinLds {
  f32x4 o[kThreads];
  float w[kJoinFew][kRowsFew];
  float m[kRowsFew], sum[kRowsFew], keep[kRowsFew];
};
// Many rows: some parts' maxima, later their weights, and sums; what the rows have so far.
constexpr int kJoinParts = 16;
struct JoinManyLds {
  float w[kJoinParts][kRowsMany], l[kJoinParts][kRowsMany];
  float m[kRowsMany], sum[kRowsMany], keep[kRowsMany];
};

template <typename T, int D, int P>
struct ChunkLds {
  using S = Shape<T, D, P>;
  union {
    char stage[2][S::STAGE];
    char own[kWaves][(S::ONE ? 1 : 2) * S::TILE];
    float o[kWaves][kRowsFew][S::OROW];
    JoinLds join;
    JoinManyLds join_many;
  } u;
  float m[kWaves][32], l[kWaves][32];
  int last;
  FindLds find;
};

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}

// 16 bytes per lane from memory at base + offset (a lane's own) to LDS at `to` +
// 16 lane, asynchronously; counted like a load.  Written out because the compiler
// waits for every copy in flight in front of any read of LDS.  (The wait states are
// those between a vector instruction that writes a scalar register and a load that
// reads it, which the compiler does not count into text of ours.)
// ONCE: not kept in the caches (16 tokens at 8K to 32K, 1.15 GB: 212 -> 196 us).
template <bool ONCE>
__device__ __forceinline__ void copy_to_lds(const void* base, uint32_t offset, uint32_t to) {
  if constexpr (ONCE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2 nt"
                 :
                 : "s"(to), "v"(offset), "s"(base)
                 : "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2"
                 :
                 : "s"(to), "v"(offset), "s"(base)
                 : "memory");
}
// until at most N of the wavefront's loads and copies are in flight
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ void barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
}

template <typename T>
__device__ __forceinline__ u32x4 lds_piece(uint32_t at) {
  return *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)at;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  uint32_t w = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
  asm("" : "+v"(w));  // one conversion for the pair: its halves are taken from w
  return w;
}

// ---- a wavefront's 32 rows -------------------------------------------------------------

template <typename T, int D, int P>
struct Rows {
  using S = Shape<T, D, P>;
  static constexpr int DT = D / 32;
  u32x4 q[S::QC];
  f32x16 acc[DT];
  float m, l;   // running maximum of the scores (unscaled) and sum of the lane's half
  int lim;      // last token that the lane's row may see
  float c;      // scale * log2(e)
  int half;
  uint32_t koff[S::QC];          // the lane's pieces of a key tile
  uint32_t voff[S::CPV / 2];     // and of a value tile's first 32 elements of d

  __device__ __forceinline__ void init(int lane, float scale) {
    half = lane >> 5;
    const int r = lane & 31;
    const int key = sizeof(T) == 2 ? (r & 16) + 8 * (r >> 2 & 1) + 4 * (r >> 3 & 1) + (r & 3) : r;
#pragma unroll
    for (int i = 0; i < S::QC; ++i)
      koff[i] = key * D * sizeof(T) + ((2 * i + half) ^ S::fk(key)) * 16;
#pragma unroll
    for (int i = 0; i < S::CPV / 2; ++i)
      voff[i] = r * P * sizeof(T) + ((2 * i + half) ^ S::fv(r)) * 16;
    c = scale * kLog2e;
  }

  __device__ __forceinline__ void start(const T* row, bool live, int limit) {
#pragma unroll
    for (int i = 0; i < S::QC; ++i)
      q[i] = live ? reinterpret_cast<const u32x4*>(row)[2 * i + half] : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;
    m = -INFINITY;
    l = 0.f;
    lim = limit;
  }

  // tiles are read from here on (LDS addresses), or `by` bytes further on
  __device__ __forceinline__ void read_from(uint32_t keys, uint32_t vals) {
#pragma unroll
    for (int i = 0; i < S::QC; ++i) koff[i] += keys;
#pragma unroll
    for (int i = 0; i < S::CPV / 2; ++i) voff[i] += vals;
  }
  __device__ __forceinline__ void move_by(uint32_t by) { read_from(by, by); }

  // S^T of the tile of keys `keys` bytes on
  __device__ __forceinline__ f32x16 scores(int keys) const {
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int i = 0; i < S::QC; ++i) {
      const u32x4 k = lds_piece<T>(keys + koff[i]);
      if constexpr (sizeof(T) == 2) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k),
                                                    __builtin_bit_cast(bf16x8, q[i]), s, 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[e]), __uint_as_float(q[i][e]), s,
                                                   0, 0, 0);
      }
    }
    return s;
  }

  // key of register e within a tile, without the lane half's part
  static __device__ constexpr int key_of(int e) {
    return sizeof(T) == 2 ? 16 * (e / 8) + e % 8 : 8 * (e / 4) + e % 4;
  }

  // Masked: keys past the lane's last one, and keys of pages that are not mapped (bit
  // i of bad: page i of the tiles).
  template <int NB>
  __device__ __forceinline__ void mask(f32x16 (&s)[NB], int key0, uint32_t bad) const {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int k = 32 * b + key_of(e) + S::E * half;
        if (key0 + k > lim || (bad >> (k / P) & 1)) s[b][e] = -INFINITY;
      }
  }

  // The running maximum with these scores; returns what to take from a score times c.
  template <int NB>
  __device__ __forceinline__ float follow(const f32x16 (&s)[NB]) {
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = b ? 0 : 1; e < 16; ++e) mx = fmaxf(mx, s[b][e]);
    mx = rows_half_max(mx);
    // The maximum follows only when a weight would pass 2^8: weights of up to 256
    // lose nothing in fp32 or bf16, and most steps leave the output as it is.
    if (wave_ballot((mx - m) * c > 8.f)) {
      const float mn = fmaxf(m, mx);
      const float alpha = __builtin_amdgcn_exp2f((m - mn) * c);
      const float a = mn == -INFINITY ? 0.f : alpha;
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] *= a;
      l *= a;
      m = mn;
    }
    return m == -INFINITY ? 0.f : m * c;
  }
  __device__ __forceinline__ float weight(float s, float mc) {
    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s, c, -mc));
    l += w;
    return w;
  }
  template <int NB>
  __device__ __forceinline__ void weights(f32x16 (&s)[NB], float mc) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[b][e] = weight(s[b][e], mc);
  }

  // The scores `next` of the tiles of keys from here on, the weights of `s` and their
  // product with the tiles of values from here on, woven together: a matrix
  // instruction takes 32 cycles of its unit and 4 to issue, so the vector
  // instructions of the softmax run beside it, a share of them behind each; LDS is
  // read four pieces ahead.  (sched_barrier: the compiler keeps this order.)  beside(i, n):
  // more to be done next to matrix instruction i of n.
  template <int NB, typename Beside>
  __device__ __forceinline__ void weave(f32x16 (&s)[NB], f32x16 (&next)[NB], float mc, Beside&& beside) {
    static_assert(sizeof(T) == 2, "tiles of many rows are bf16");
    constexpr int SE = 16 / (32 / (2 * S::E));   // scores of a lane that a step of values takes
    constexpr int NS = NB * S::QC, STEPS = NB * 16 / SE, TOTAL = NS + STEPS * DT;
    constexpr int AHEAD = 4, EL = NB * 16, SPAN = TOTAL - DT;
    u32x4 buf[AHEAD + 1];
    bf16x8 w;
    auto fetch = [&](int i) {
      if (i < NS) return lds_piece<T>(koff[i / NB] + i % NB * S::TILE);
      const int st = (i - NS) / DT, dt = (i - NS) % DT;          // step, 32 elements of d
      const int piece = 2 * (st % (STEPS / NB)), tile = st / (STEPS / NB);
      return lds_piece<T>(voff[piece % S::CPV / 2] +
                          (tile * S::TILE + piece / S::CPV * (int)(D * P * sizeof(T)) +
                           dt * (int)(32 * P * sizeof(T))));
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) buf[i] = fetch(i);
#pragma unroll
    for (int i = 0; i < TOTAL; ++i) {
      if (i + AHEAD < TOTAL) buf[(i + AHEAD) % (AHEAD + 1)] = fetch(i + AHEAD);
      const u32x4 x = buf[i % (AHEAD + 1)];
      if (i < NS) {
        f32x16& n = next[i % NB];
        if (i < NB)
#pragma unroll
          for (int e = 0; e < 16; ++e) n[e] = 0.f;
        n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x),
                                                    __builtin_bit_cast(bf16x8, q[i / NB]), n, 0, 0, 0);
      } else {
        const int st = (i - NS) / DT, dt = (i - NS) % DT, e0 = st * SE;
        if (dt == 0) {
          u32x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            y[e] = pack_bf16(s[e0 / 16][e0 % 16 + 2 * e], s[e0 / 16][e0 % 16 + 2 * e + 1]);
          w = __builtin_bit_cast(bf16x8, y);
        }
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), w, acc[dt], 0, 0, 0);
      }
#pragma unroll
      for (int e = min(i * EL / SPAN, EL); e < min((i + 1) * EL / SPAN, EL); ++e)
        s[e / 16][e % 16] = weight(s[e / 16][e % 16], mc);
      beside(i, TOTAL);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // Zeroes an fp32 tile's values of slots that hold no token of the sequence (stored:
  // tokens of it from this tile's first key on), each lane those that it will read.
  __device__ __forceinline__ void clear(int stored, uint32_t bad) const {
#pragma unroll
    for (int piece = 0; piece < 32 / S::E; piece += 2) {
      const int k = S::E * (piece + half), n = bad >> (k / P) & 1 ? 0 : stored - k;
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const uint32_t at = voff[piece % S::CPV / 2] + (piece / S::CPV * D + i * 32) * P * sizeof(T);
        u32x4 v = lds_piece<T>(at);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = n > e ? v[e] : 0u;
        *(__attribute__((address_space(3))) u32x4*)(uintptr_t)at = v;
      }
    }
  }

  // O^T += V^T P^T of one tile.  bf16 values of slots that hold no token are taken as
  // zero here: an AND beside each of few matrix instructions, hidden by the memory
  // (fp32, with four times as many and each four times as long, would wait for them:
  // 1024 rows at 1024, d 128, 370 -> 328 us without).
  // SPLIT: a bf16 weight is given as two, what the first one's rounding leaves and it.
  // Tiles of many rows, bound by the matrix units, take the rounded one alone: with
  // both 8192 rows 502 -> 690 us and 1024 at 131K 1857 -> 2593, for outputs of 2000 rows
  // 1.9e-4 -> 1.5e-4 off 64 bits (root mean squares; of the outputs 0.09).
  template <bool SPLIT>
  __device__ __forceinline__ void values(int at, const f32x16& p, int stored, uint32_t bad) {
    constexpr int STEPS = 32 / (2 * S::E);  // key pieces of a lane half
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      const int piece = 2 * t;  // (+ half) of the tile; pieces of a page: CPV
      const int more = at + piece / S::CPV * (int)(D * P * sizeof(T));
      [[maybe_unused]] bf16x8 w, rest;
      if constexpr (sizeof(T) == 2) {
        u32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = pack_bf16(p[8 * t + 2 * e], p[8 * t + 2 * e + 1]);
        w = __builtin_bit_cast(bf16x8, x);
        if constexpr (SPLIT) {
          u32x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            y[e] = pack_bf16(p[8 * t + 2 * e] - __uint_as_float(x[e] << 16),
                             p[8 * t + 2 * e + 1] - __uint_as_float(x[e] & 0xffff0000u));
          rest = __builtin_bit_cast(bf16x8, y);
        }
      }
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        u32x4 v = lds_piece<T>(voff[piece % S::CPV / 2] + (more + i * (int)(32 * P * sizeof(T))));
        const int k = S::E * (piece + half);
        [[maybe_unused]] const int n = bad >> (k / P) & 1 ? 0 : stored - k;  // elements that count
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[e] &= (n > 2 * e ? 0xffffu : 0u) | (n > 2 * e + 1 ? 0xffff0000u : 0u);
          acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), w, acc[i], 0,
                                                           0, 0);
          if constexpr (SPLIT)
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), rest, acc[i],
                                                             0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(v[e]), p[4 * t + e], acc[i],
                                                          0, 0, 0);
        }
      }
    }
  }
};

template <typename T>
__device__ __forceinline__ void store4(T* p, float a, float b, float c, float d) {
  if constexpr (sizeof(T) == 2) {
    uint2 w;
    w.x = pack_bf16(a, b);
    w.y = pack_bf16(c, d);
    *reinterpret_cast<uint2*>(p) = w;
  } else {
    *reinterpret_cast<f32x4*>(p) = f32x4{a, b, c, d};
  }
}

__device__ __forceinline__ float natural_lse(float m, float l, float scale) {
  return l == 0.f ? -INFINITY : __builtin_fmaf(m, scale, __builtin_amdgcn_logf(l) * kLn2);
}

// A sequence's pages: page i's number if it is mapped, else page 0 (never counted).
struct Pages {
  const int32_t* table;
  int last, num_phys;
  __device__ __forceinline__ int operator()(int i, bool& bad) const {
    const int id = sload(table + min(i, last));
    bad = id < 0 || id >= num_phys;
    return bad ? 0 : id;
  }
  // pages without a mapping among n (those past the end are cut by lengths)
  template <int N>
  __device__ __forceinline__ uint32_t bad(int page0) const {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      bool b;
      (*this)(page0 + i, b);
      bits |= (uint32_t)b << i;
    }
    return bits;
  }
};

// A sequence's pages, and row rho of its rows for KV head h (the last one for those behind it).
template <int P>
__device__ __forceinline__ Pages pages_of(const AttendCall& a, const Seq& s, int b) {
  return Pages{a.pt + (int64_t)b * a.max_pages, max((s.end + P - 1) / P - 1, 0), a.num_phys};
}
template <typename T, int D>
__device__ __forceinline__ const T* row_at(const AttendCall& a, const Seq& s, int h, int rho, bool& live, int& lim) {
  live = rho < s.rows;
  const int r = min(rho, s.rows - 1);
  lim = min(s.run.pos + r / a.G, s.end - 1);
  return (const T*)a.q + (int64_t)(s.run.row + r / a.G) * a.q_stride + (int64_t)(h * a.G + r % a.G) * D;
}

// ---- parts -------------------------------------------------------------------------------

// Stores and loads of parts go past the XCDs' L2s, through a resource per part.
__device__ __forceinline__ void put_part(__amdgpu_buffer_rsrc_t r, int at, f32x4 v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4v, v), r, at * 4, 0, kCpolSc1);
}
__device__ __forceinline__ void put_part(__amdgpu_buffer_rsrc_t r, int at, float v) {
  __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r, at * 4, 0, kCpolSc1);
}

// Whether this workgroup is the last of `parts` to come here; its stores and the others' are then done.
__device__ __forceinline__ bool last_part(int32_t* counter, int parts, int* flag, int tid) {
  __builtin_amdgcn_s_waitcnt(0);  // this wavefront's stores have been acknowledged
  __syncthreads();
  if (tid == 0) {
    const int n = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (n == parts - 1) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = n == parts - 1;
  }
  __syncthreads();
  return *flag != 0;
}

// Joins the parts of R of a tile's 32 rows: slot(p) is part p's result.  16 lanes a
// row take the maxima and sums of 64 parts; then all threads the outputs, 16 bytes
// each, where there are fewer rows than threads for it several groups of them a
// share of the parts each.  done(row, m, l, d, o): four elements from d on.
template <int D, typename Slot, typename Done>
__device__ __forceinline__ void join_few(JoinLds& L, int R, int parts, float c, int tid, Slot&& slot,
                                         Done&& done) {
  constexpr int LPR = D / 4, PER = kThreads / LPR;       // rows at a time
  constexpr int ITEMS = kRowsFew / PER;                  // rows of a thread: row0 + i * PER
  const int d = tid % LPR * 4, sub = tid / LPR;
  int shift = 0;                                         // 2^shift groups share the parts
  while ((R << (shift + 1)) <= PER) ++shift;
  const int groups = 1 << shift, grp = sub & (groups - 1), row0 = sub >> shift;
  f32x4 o[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (tid < kRowsFew) {
    L.m[tid] = -INFINITY;
    L.sum[tid] = 0.f;
  }
  __syncthreads();
  constexpr int AHEAD = 8;
  f32x4 x[AHEAD][ITEMS];
  auto load = [&](int q0, int np, int p0) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const __amdgpu_buffer_rsrc_t r = coherent_rsrc(slot(q0));
      const int at = (int)((const char*)slot(q0 + min(p0 + j * groups, np - 1)) - (const char*)slot(q0));
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
        x[j][i] = __builtin_bit_cast(
            f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                       r, at + (min(row0 + i * PER, R - 1) * D + d) * 4, 0, kCpolSc1));
    }
  };
  for (int q0 = 0; q0 < parts; q0 += kJoinFew) {
    const int np = min(parts - q0, kJoinFew);
    load(q0, np, grp);  // on the way while the weights are made
    {
      const int row = tid / 16, j = tid % 16;  // kThreads / 16 == kRowsFew
      float pm[kJoinFew / 16], pl[kJoinFew / 16];
#pragma unroll
      for (int i = 0; i < kJoinFew / 16; ++i) {
        const int p = j + 16 * i;
        const __amdgpu_buffer_rsrc_t r = coherent_rsrc(slot(q0));
        // (a part's place behind the first one's, in bytes)
        const int at = (int)((const char*)slot(q0 + min(p, np - 1)) - (const char*)slot(q0));
        pm[i] = __uint_as_float(
            __builtin_amdgcn_raw_buffer_load_b32(r, at + (kRowsFew * D + row) * 4, 0, kCpolSc1));
        pl[i] = __uint_as_float(
            __builtin_amdgcn_raw_buffer_load_b32(r, at + (kRowsFew * (D + 1) + row) * 4, 0, kCpolSc1));
        if (p >= np || row >= R) pm[i] = -INFINITY;
      }
      float m = L.m[row];
#pragma unroll
      for (int i = 0; i < kJoinFew / 16; ++i) m = fmaxf(m, pm[i]);
      m = fmaxf(m, dpp_f<kDppXor1>(m));
      m = fmaxf(m, dpp_f<kDppXor2>(m));
      m = fmaxf(m, dpp_f<kDppHalfMirror>(m));
      m = fmaxf(m, dpp_f<kDppMirror>(m));
      const float mu = m == -INFINITY ? 0.f : m, keep = __builtin_amdgcn_exp2f((L.m[row] - mu) * c);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kJoinFew / 16; ++i) {
        const int p = j + 16 * i;
        const float w = __builtin_amdgcn_exp2f((pm[i] - mu) * c);
        if (p < np) {
          sum = __builtin_fmaf(w, row < R ? pl[i] : 0.f, sum);
          L.w[p][row] = w;
        }
      }
      sum += dpp_f<kDppXor1>(sum);
      sum += dpp_f<kDppXor2>(sum);
      sum += dpp_f<kDppHalfMirror>(sum);
      sum += dpp_f<kDppMirror>(sum);
      if (j == 0) {
        L.sum[row] = __builtin_fmaf(L.sum[row], keep, sum);
        L.m[row] = m;
        L.keep[row] = keep;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] *= L.keep[min(row0 + i * PER, R - 1)];
    for (int p0 = grp; p0 < np; p0 += AHEAD * groups) {
      if (p0 != grp) load(q0, np, p0);
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        if (p0 + j * groups >= np) continue;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
          const float w = L.w[p0 + j * groups][min(row0 + i * PER, R - 1)];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][e] = __builtin_fmaf(w, x[j][i][e], o[i][e]);
        }
      }
    }
    __syncthreads();
  }
  if (groups > 1) {  // (then R <= PER, and a thread has one row)
    L.o[tid] = o[0];
    __syncthreads();
    if (grp == 0)
      for (int g = 1; g < groups; ++g) {
        const f32x4 y = L.o[tid + g * LPR];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[0][e] += y[e];
      }
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int row = row0 + i * PER;
    if (grp == 0 && row < R) done(row, L.m[row], L.sum[row], d, o[i]);
  }
}

// The same for up to 256 rows: a slot is read by all threads at once, 16 bytes of up
// to 16 rows each (D 128), which keeps 128 KB on the way.  (Row after row, eight parts
// at a time, nine parts of 256 rows took 100 us: the loads go to memory.)
template <int D, typename Slot, typename Done>
__device__ __forceinline__ void join_many(JoinManyLds& L, int R, int parts, float c, int tid,
                                          Slot&& slot, Done&& done) {
  constexpr int ITEMS = kRowsMany * (D / 4) / kThreads, PER = kThreads / (D / 4);
  const int row0 = tid / (D / 4), d = tid % (D / 4) * 4;  // rows row0 + i * PER
  f32x4 o[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (tid < kRowsMany) {
    L.m[tid] = -INFINITY;
    L.sum[tid] = 0.f;
  }
  for (int q0 = 0; q0 < parts; q0 += kJoinParts) {
    const int np = min(parts - q0, kJoinParts);
    for (int i = tid; i < np * kRowsMany; i += kThreads) {
      const int p = i / kRowsMany, row = i % kRowsMany;
      if (row >= R) continue;
      const __amdgpu_buffer_rsrc_t r = coherent_rsrc(slot(q0 + p));
      L.w[p][row] = __uint_as_float(
          __builtin_amdgcn_raw_buffer_load_b32(r, (kRowsMany * D + row) * 4, 0, kCpolSc1));
      L.l[p][row] = __uint_as_float(
          __builtin_amdgcn_raw_buffer_load_b32(r, (kRowsMany * (D + 1) + row) * 4, 0, kCpolSc1));
    }
    __syncthreads();
    if (tid < R) {
      float m = L.m[tid];
      for (int p = 0; p < np; ++p) m = fmaxf(m, L.w[p][tid]);
      const float mu = m == -INFINITY ? 0.f : m, keep = __builtin_amdgcn_exp2f((L.m[tid] - mu) * c);
      float sum = L.sum[tid] * keep;
      for (int p = 0; p < np; ++p) {
        const float w = __builtin_amdgcn_exp2f((L.w[p][tid] - mu) * c);
        sum = __builtin_fmaf(w, L.l[p][tid], sum);
        L.w[p][tid] = w;
      }
      L.m[tid] = m;
      L.sum[tid] = sum;
      L.keep[tid] = keep;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] *= row0 + i * PER < R ? L.keep[row0 + i * PER] : 0.f;
    for (int p = 0; p < np; ++p) {
      const __amdgpu_buffer_rsrc_t r = coherent_rsrc(slot(q0 + p));
      f32x4 x[ITEMS];
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int row = min(row0 + i * PER, R - 1);
        x[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (row * D + d) * 4, 0, kCpolSc1));
      }
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const float w = L.w[p][min(row0 + i * PER, R - 1)];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][j] = __builtin_fmaf(w, x[i][j], o[i][j]);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int row = row0 + i * PER;
    if (row < R) done(row, L.m[row], L.sum[row], d, o[i]);
  }
}

// ---- many rows ---------------------------------------------------------------------------

// Stages of 64 keys for all wavefronts, copied from pages in T.
template <typename T, int D, int P>
struct CopiedStages {
  using S = Shape<T, D, P>;
  static constexpr int MINE = S::NB * S::LOADS / kWaves;  // copies of keys (and of values) per wavefront
  static_assert(MINE >= 1 && S::PPP % MINE == 0, "a wavefront's copies lie in one page");
  int64_t phys_bytes, page_bytes;
  uint32_t kcopy, vcopy;  // a lane's place within a copy of keys, and of values
  const char *kh, *vh;
  Pages page_of;
  uint32_t to;
  int first, page, page_next;

  __device__ __forceinline__ int page_at(int key) const {  // of the wavefront's copies of the stage from this key on
    bool bad;
    return page_of(key / P + first / S::PPP, bad);
  }
  // copy i of a tile: rows further on, whose numbers change the order by this
  static __device__ __forceinline__ uint32_t kxor(int i) { return (uint32_t)S::fk(i * (64 / S::CPR) & 31) << 4; }
  static __device__ __forceinline__ uint32_t vxor(int i) { return S::CPV == 8 ? (uint32_t)(i & 1) << 6 : 0u; }
  __device__ __forceinline__ void copy_keys(int page) {
    const char* src = kh + page * phys_bytes + first % S::PPP * 1024;
#pragma unroll
    for (int i = 0; i < MINE; ++i)
      copy_to_lds<false>(src + i * 1024, kcopy ^ kxor(first + i), to + (first + i) * 1024);
  }
  __device__ __forceinline__ void copy_values(int page) {
    const char* src = vh + page * phys_bytes + first % S::PPP * 1024;
#pragma unroll
    for (int i = 0; i < MINE; ++i)
      copy_to_lds<false>(src + i * 1024, vcopy ^ vxor(first + i), to + S::NB * S::TILE + (first + i) * 1024);
  }
  // a tile of KV head h begins; LDS stages from `st` on
  __device__ __forceinline__ void start(const AttendCall& a, const Pages& pages, int h, uint32_t st, int wave) {
    page_of = pages;
    kh = (const char*)a.kc + h * page_bytes;
    vh = (const char*)a.vc + h * page_bytes;
    to = st;
    first = wave * MINE;
  }
  // the first stage's keys are there when this returns, its values and the next keys on their way
  __device__ __forceinline__ void begin(int key, int key_end, int32_t by) {
    page = page_at(key);
    page_next = page_at(key + S::KEYS);
    copy_keys(page);
    to += by;
    copy_values(page);
    if (key + S::KEYS < key_end) copy_keys(page_next);
    page = page_next;
    page_next = page_at(key + 2 * S::KEYS);
    wait_loads<MINE>();
    barrier();
  }
  // in front of the work on the stage at `key`: its copies are there, the next one's begin
  __device__ __forceinline__ void turn(int key, int key_end, int32_t by) {
    wait_loads<0>();
    barrier();
    to += by;
    if (key + S::KEYS < key_end) copy_values(page);
    if (key + 2 * S::KEYS < key_end) copy_keys(page_next);
    page = page_next;
    page_next = page_at(key + 3 * S::KEYS);
  }
  // what is left of a turn: beside the matrix instructions, or at once
  __device__ __forceinline__ void beside(int, int) {}
  __device__ __forceinline__ void finish() {}
};

// Tiles of 256 rows: 32 of them for each wavefront, over the same 64 keys.  finish: the
// result of a row, four elements of d.
template <typename T, int D, int P, typename Lds, typename Stages, typename Finish>
__device__ __forceinline__ void many_rows(const AttendCall& a, const Cut& cut, Lds& L, int tid, int wave,
                                          Stages stages, Finish&& finish) {
  using S = Shape<T, D, P>;
  using R_t = Rows<T, D, P>;
  const uint32_t st = lds_address(&L.u);
  constexpr int PS = S::KEYS / P;  // pages of a stage
  const int most = (int)cut.part;
  auto parts_of = [&](int steps) { return (steps + most - 1) / most; };
  for (int64_t round = 0;; ++round) {
    // longest first; every other round backwards, eight neighbours (one per XCD) together
    int64_t k = blockIdx.x;
    if (round & 1) k = (int64_t)(gridDim.x / 8 - 1 - k / 8) * 8 + k % 8;
    int b;
    int64_t u, before;
    Seq s;
    if (!find_seq(a, P, round * gridDim.x + k, L.find, tid,
                  [&](const Seq& s) {
                    return s.few ? 0 : (int64_t)s.tiles(kRowsMany) * a.hk * parts_of(s.steps());
                  },
                  [&](const Seq& s) {
                    return s.few || s.steps() <= most
                               ? 0
                               : (int64_t)s.tiles(kRowsMany) * a.hk * parts_of(s.steps());
                  },
                  s, b, u, before))
      break;
    const int un = __builtin_amdgcn_readfirstlane((int)u);
    // KV head fastest (a head's units meet in one L2), then row tiles, last first
    const int tiles = s.tiles(kRowsMany);
    const int h = un % a.hk, part = un / a.hk / tiles, back = un / a.hk % tiles;
    const int tile = tiles - 1 - back;
    const int R = min(s.rows - tile * kRowsMany, kRowsMany);
    const int end = s.seen(tile * kRowsMany + R, a.G);   // tokens that the tile sees
    const int steps = max((end + 63) / 64, 1), parts = parts_of(steps);
    if (part >= parts) continue;
    const int per = (steps + parts - 1) / parts;
    const int key_begin = part * per * 64, key_end = min(end, (part + 1) * per * 64);
    const Pages page_of = pages_of<P>(a, s, b);
    const int lane = thread_index() & 63;
    R_t rows;
    rows.init(lane, a.scale);
    const int rho0 = tile * kRowsMany + wave * 32;
    const bool any = rho0 < s.rows;
    bool live;
    int lim;
    const T* qrow = row_at<T, D>(a, s, h, rho0 + (lane & 31), live, lim);
    rows.start(qrow, live, lim);
    rows.read_from(st, st + S::NB * S::TILE);
    // Every row sees the tokens up to the first row's; stages behind them, and all
    // where a page is not mapped, are masked.  No row of the wavefront sees past lim1.
    const int np = (key_end + P - 1) / P;
    bool missing = false;
    for (int i = key_begin / P + tid; i < np; i += kThreads) {
      const int id = page_of.table[i];
      missing |= id < 0 || id >= a.num_phys;
    }
    const int seen = __syncthreads_or(missing) ? 0 : min(s.run.pos + tile * kRowsMany / a.G, s.end - 1) + 1;
    const int lim1 =
        any ? min(s.run.pos + min(rho0 + 31, s.rows - 1) / a.G, s.end - 1) : -1;
    // A stage of LDS holds 64 keys' values and the next 64 keys: while the weights of
    // one are taken, the scores of the next are made.
    int key = key_begin;
    int32_t by = S::STAGE;  // to the other stage
    stages.start(a, page_of, h, st, wave);
    auto turn = [&]() { stages.turn(key, key_end, by); };
    auto next_stage = [&]() {
      rows.move_by(by);
      by = -by;
      key += S::KEYS;
    };
    if (key_begin < key_end) {
      f32x16 sa[S::NB], sb[S::NB];
      stages.begin(key, key_end, by);
#pragma unroll
      for (int i = 0; i < S::NB; ++i) sa[i] = rows.scores(i * S::TILE);
      rows.move_by(by);
      by = -by;
      // stages that no mask touches, up to the last but one
      const int clean = min(seen / S::KEYS * S::KEYS, key_end - S::KEYS);
      auto step = [&](f32x16(&cur)[S::NB], f32x16(&next)[S::NB]) {
        turn();
        rows.weave(cur, next, rows.follow(cur), [&](int i, int n) { stages.beside(i, n); });
        next_stage();
      };
      while (key + S::KEYS < clean) {
        step(sa, sb);
        step(sb, sa);
      }
      if (key < clean) {
        step(sa, sb);
#pragma unroll
        for (int i = 0; i < S::NB; ++i) sa[i] = sb[i];
      }
      while (key < key_end) {
        turn();
        stages.finish();
        if (key <= lim1) {
          const uint32_t bad = page_of.template bad<PS>(key / P);
          rows.mask(sa, key, bad);
          rows.weights(sa, rows.follow(sa));
#pragma unroll
          for (int i = 0; i < S::NB; ++i)
            rows.template values<false>(i * S::TILE, sa[i], s.end - key - 32 * i, bad >> (i * 32 / P));
        }
        if (key + S::KEYS <= lim1)
#pragma unroll
          for (int i = 0; i < S::NB; ++i) sa[i] = rows.scores(i * S::TILE);
        next_stage();
      }
    }
    rows.l = rows_half_sum(rows.l);
    const int rt = wave * 32 + (lane & 31);
    auto slot = [&](int p) {
      return a.many + (before + ((int64_t)p * tiles + back) * a.hk + h) * slot_floats(kRowsMany, D);
    };
    const __amdgpu_buffer_rsrc_t dst = coherent_rsrc(slot(part));
    if (rt < R) {
#pragma unroll
      for (int i = 0; i < R_t::DT; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const int d = i * 32 + 2 * e + 4 * rows.half;
          const f32x4 o{rows.acc[i][e], rows.acc[i][e + 1], rows.acc[i][e + 2], rows.acc[i][e + 3]};
          if (parts > 1) put_part(dst, rt * D + d, o);
          else finish(s, h, tile * kRowsMany + rt, rows.m, rows.l, d, o);
        }
      if (parts > 1 && lane < 32) {
        put_part(dst, kRowsMany * D + rt, rows.m);
        put_part(dst, kRowsMany * (D + 1) + rt, rows.l);
      }
    }
    if (parts > 1) {
      const int64_t first = before + (int64_t)back * a.hk + h;  // the tile's first part among all
      if (last_part(a.counters + kCus + first, parts, &L.last, tid))
        join_many<D>(L.u.join_many, R, parts, rows.c, tid, slot,
                     [&](int row, float m, float l, int d, f32x4 o) {
                       finish(s, h, tile * kRowsMany + row, m, l, d, o);
                     });
    }
    barrier();
  }
}

}  // namespace
}  // namespace retro
