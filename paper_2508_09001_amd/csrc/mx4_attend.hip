// Dense causal attention of a ragged batch of rows over a paged cache in 4 bits: what
// chunk_attend.hip does over pages in dtype, with the same layout of the work
// (chunk_work.h): the steps of all tiles of 32 rows form one line, cut into shares for
// the workgroups, and the parts of a cut tile are joined by the workgroup that counts
// itself last; tiles of 256 rows where there is work for them (bf16).
//   - 32 rows: a workgroup's wavefronts take 32 tokens in turn, codes straight from the page into
//     registers (mx4_rows.h), and join their (maximum, sum, output) at the end of a tile.  Up to 16
//     rows are one tile of a product, of which more wavefronts' instructions are left.
//   - 256 rows: chunk_attend.hip's stages of 64 keys in LDS, in bf16, which the wavefronts
//     make of the codes while they work on the stage in front (Mx4Stages).
//
// Measured (bf16, 8 KV heads of 4 query heads of 128): 16 tokens at 8K to 32K, 306 MB of
// codes, 62 us (187 over pages in bf16): 50 of them at 6.1 TB/s, the rest is the first keys' way and
// the joins; a token at 32768 18.0 us (32.5), of which 4.6 are the reading, 1.6 the start of all
// workgroups, 3.8 lengths, layout and page numbers, 1.9 the slowest wavefront's lead, 1.2 the
// joining of eight wavefronts and 4 that of 32 parts.  8192 rows from 0 512 to 571 us on cards
// where pages in bf16 take 486 to 520 (91 to 95 % of their rate): the matrix units are busy 48 % of the cycles, the vector
// units, which do the softmax and the conversion, 57 %. Two workgroups of a compute unit side by
// side, with half of the registers and 512 shares, took 82 us for the 16 tokens and 34 for the one,
// whose 64 parts are joined by one workgroup.
#include "chunk_work.h"
#include "mx4_rows.h"

namespace retro {
namespace {

// What a wavefront reads of a stage of 64 keys: codes and exponents of eight tokens' keys,
// and of eight tokens' values.
template <int D>
struct Mx4Share {
  char codes[2][4 * D], exps[2][D / 4];
};

template <int D, int P, bool MANY>
struct Mx4Lds {
  using S = Shape<bf16_t, D, P>;
  static constexpr int OROW = D + 4;
  union {
    struct {
      char stage[2][MANY ? S::STAGE : 16];
      Mx4Share<D> shares[MANY ? 2 * kWaves : 1];
    } many;
    float o[kWaves][kRowsFew][OROW];
    JoinLds join;
    JoinManyLds join_many;
  } u;
  float m[kWaves][kRowsFew], l[kWaves][kRowsFew];
  int last;
  FindLds find;
};

// Stages of 64 keys for tiles of many rows, as chunk_attend.hip's copies leave them in LDS.
// Each wavefront copies an eighth of the next stage's codes to LDS (eight tokens of one
// page, keys and values), converts those of this one to bf16, values with eight tokens of
// an element together, and writes them to the stage.  The conversion is woven into the
// matrix instructions of the stage in front.
template <int D, int P>
struct Mx4Stages {
  using S = Shape<bf16_t, D, P>;
  static constexpr int64_t kBlock = mx4_block_bytes(P, D);
  static constexpr int KP = D / 64;  // 16-byte pieces of a key that a lane makes
  const Mx4Share<D>* shares;         // the workgroup's, of two stages
  int64_t phys_bytes;
  const char *kh, *vh;
  Pages page_of;
  uint32_t to;
  int wave, now, page_k, page_v;  // share that is converted next; pages to be copied next
  uint32_t k[KP], ke, v[2][D / 32], ve[2], x[8];
  // where the lane reads a share and writes a stage, two places to a register (the loop has
  // few left: places worked out in it cost as many instructions as the conversion, kept apart they
  // are spilled): codes and exponent of keys, of values; its piece of a key, of a value
  uint32_t of_keys, of_values, puts;

  __device__ __forceinline__ int page_at(int key) const {
    bool bad;
    return page_of((key + 8 * wave) / P, bad);
  }
  __device__ __forceinline__ const Mx4Share<D>& share(int which) const { return shares[which * kWaves + wave]; }
  // copies keys of one page and values of another into a share, without waiting
  __device__ __forceinline__ void copy(int key_page, int value_page, const Mx4Share<D>& s) const {
    const int lane = thread_index() & 63, slot = 8 * wave % P;
    const char *kb = kh + key_page * phys_bytes, *vb = vh + value_page * phys_bytes;
    // (m0 and its wait states as in copy_to_lds)
    if (lane < D / 2) {
      const char* from = (lane < D / 4 ? kb : vb) + (slot * (D / 2) + (lane & (D / 4 - 1)) * 16);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, off"
                   :
                   : "s"(__builtin_amdgcn_readfirstlane(lds_address(s.codes))), "v"(from)
                   : "memory");
    }
    if (lane < D / 8) {
      const char* from = (lane < D / 16 ? kb : vb) + (P * D / 2 + slot * (D / 32) + (lane & (D / 16 - 1)) * 4);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, off"
                   :
                   : "s"(__builtin_amdgcn_readfirstlane(lds_address(s.exps))), "v"(from)
                   : "memory");
    }
  }
  // the next copy: values of the stage at `key` and the keys behind them
  __device__ __forceinline__ void copy_next(int key, int key_end) {
    if (key < key_end) copy(page_k, page_v, share(now ^ 1));
    page_v = page_k;
    page_k = page_at(key + 2 * S::KEYS);
  }
  __device__ __forceinline__ void places() {
    const int lane = thread_index() & 63, part = lane / (D / 32) & 15;
    of_keys = lane * (D / 16) | (lane / 8 * (D / 32) + lane % 8 * (D / 8) / 32) << 16;
    of_values = part * (D / 8) | (lane / 16) % (D / 32) * 4 << 16;
    const int key = 8 * wave + lane / 8, row = key % 32, token = 8 * wave % 32, d = 2 * lane % D;
    const int at_key = key / 32 * S::TILE + row * (D * 2) + (lane % 8 * KP ^ S::fk(row)) * 16;
    const int at_value = 8 * wave / 32 * S::TILE + token / P * (D * P * 2) + (d + (lane >> 3 & 1)) * (P * 2) +
                         (token % P / 8 ^ S::fv(d)) * 16;
    static_assert(S::NB * S::TILE <= 1 << 16, "places within a stage's keys, or values, have 16 bits");
    puts = at_key | at_value << 16;
    asm volatile("" : "+v"(of_keys), "+v"(of_values), "+v"(puts));  // kept as they are
  }
  // the lane's part of the share
  __device__ __forceinline__ void read() {
    const uint32_t s = lds_address(&share(now));
    auto word = [](uint32_t at) { return *(const __attribute__((address_space(3))) uint32_t*)(uintptr_t)at; };
    const uint32_t at_k = s + (of_keys & 0xffff), at_v = s + 4 * D + (of_values & 0xffff);
#pragma unroll
    for (int i = 0; i < KP; ++i) k[i] = word(at_k + 4 * i);
    ke = *(const __attribute__((address_space(3))) uint8_t*)(uintptr_t)(s + 8 * D + (of_keys >> 16));
    // elements 2 lane, 2 lane + 1 of eight tokens
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < D / 32; ++i) v[t][i] = word(at_v + t * (2 * D) + 4 * i);
      ve[t] = word(s + 8 * D + D / 4 + (of_values >> 16) + t * (D / 8));
    }
  }
  static __device__ __forceinline__ void put(uint32_t at, u32x4 y) {
    *(__attribute__((address_space(3))) u32x4*)(uintptr_t)at = y;
  }
  __device__ __forceinline__ void put_keys(int i) const {
    // (a lane's pieces are neighbours, the first of even number: their places differ in one bit)
    put(to + ((puts & 0xffff) ^ 16 * i), mx4_piece<bf16_t>(k[i], mx4_scale((int)ke)));
  }
  __device__ __forceinline__ void convert_values(int t, int e) {
    // (a scale's bits below its exponent field, and its sign, do not count)
    const float scale = __uint_as_float(e < 3 ? ve[t] << (23 - 8 * e) : ve[t] >> 1);
    const uint32_t w = v[t][e * (D / 32) / 4] >> (of_keys * (128 / D) & (D / 32 - 1) * 8);  // byte lane % (D / 32)
    x[4 * t + e] = e * (D / 32) % 4 ? mx4_bf16<2>(w, scale) : mx4_bf16<0>(w, scale);
  }
  // One of a lane's two elements, then the other: every other eight lanes begin with the second
  // one, so that sixteen write to as many groups of banks.  (Element d + 1 has the order of
  // pieces of element d; for d 64 two lanes write the same.)
  __device__ __forceinline__ void put_values(int other) const {
    constexpr int kRow = P * 2;  // bytes of an element's tokens in a page
    const uint32_t halves = (0x05040100u + (puts >> 16 & kRow) / kRow * 0x02020202u) ^ other * 0x02020202u;
    u32x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], halves);
    put(to + S::NB * S::TILE + (puts >> 16 ^ other * kRow), y);
  }
  // the conversion in kUnits units
  static constexpr int kUnits = 11 + KP;
  __device__ __forceinline__ void unit(int u) {
    if (u == 0) read();
    else if (u <= KP) put_keys(u - 1);
    else if (u <= KP + 8) convert_values((u - KP - 1) / 4, (u - KP - 1) % 4);
    else put_values(u - KP - 9);
  }
  // (from the first product's last instructions on: 8192 rows from 0 547 us spread over all of
  // them, 543, 541, 541, 544 and 549 from number 4, 8, 12, 16 and 20 of 32 on; without the
  // conversion 10 % less, of which values, with their shifts and halves, are two thirds)
  __device__ __forceinline__ void beside(int i, int n) {
    const int first = n * 3 / 8;
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
      if (u * (n - first) / kUnits + first == i) unit(u);
  }
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) unit(u);
  }
  __device__ __forceinline__ void start(const AttendCall& a, const Pages& pages, int h, uint32_t st, int w) {
    page_of = pages;
    phys_bytes = kBlock * a.hk;
    kh = (const char*)a.kc + h * kBlock;
    vh = (const char*)a.vc + h * kBlock;
    to = st;
    wave = w;
    places();
  }
  // the first stage of LDS takes the first keys, the second one their values and the next keys
  __device__ __forceinline__ void begin(int key, int key_end, int32_t by) {
    page_v = page_at(key);
    page_k = page_at(key + S::KEYS);
    copy(page_v, page_v, share(0));
    copy(page_k, page_v, share(1));
    wait_loads<0>();
    now = 0;
    read();
#pragma unroll
    for (int i = 0; i < KP; ++i) put_keys(i);
    to += by;
    now = 1;
    finish();
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    page_v = page_k;
    page_k = page_at(key + 2 * S::KEYS);
    copy_next(key + S::KEYS, key_end);
    barrier();
  }
  // in front of the work on the stage at `key`, which is there: the next one's codes are
  // there too, and those behind them are copied (what is converted past the end is not used)
  __device__ __forceinline__ void turn(int key, int key_end, int32_t by) {
    wait_loads<0>();
    barrier();
    to += by;
    now ^= 1;
    copy_next(key + 2 * S::KEYS, key_end);
  }
};

// MANY: with tiles of many rows, as in chunk_attend.hip.
template <typename T, int D, int P, bool MANY>
__global__ void __launch_bounds__(kThreads) mx4_attend_kernel(AttendCall a) {
  __shared__ __attribute__((aligned(1024))) Mx4Lds<D, P, MANY> L;
  const int tid = thread_index();
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Cut cut = make_cut<MANY, true>(a, P, L.find, tid);
  constexpr int64_t kBlock = mx4_block_bytes(P, D);
  const int64_t phys_bytes = kBlock * a.hk;
  const float c = a.scale * kLog2e;

  // the result of row rho of a sequence's rows for KV head h, four elements of d
  auto finish = [&](const Seq& s, int h, int rho, float m, float l, int d, f32x4 o) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t at = (int64_t)(s.run.row + rho / a.G) * a.hq + h * a.G + rho % a.G;
    store4((T*)a.out + at * D + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    if (d == 0 && a.lse) a.lse[at] = natural_lse(m, l, a.scale);
  };

  // The rows from rho0 on (nr of them) with the keys of [key_begin, key_end), this
  // wavefront's share of them; results into LDS.
  auto tile_of = [&](auto row_tiles, const Seq& s, int b, int h, int rho0, int nr, int begin, int end) {
    constexpr int NR = decltype(row_tiles)::value;
    const int lane = thread_index() & 63;
    const int key_begin = __builtin_amdgcn_readfirstlane(begin), key_end = __builtin_amdgcn_readfirstlane(end);
    const Pages page_of{a.pt + (int64_t)b * a.max_pages, max((s.end + P - 1) / P - 1, 0), a.num_phys};
    const char* kh = (const char*)a.kc + h * kBlock;
    const char* vh = (const char*)a.vc + h * kBlock;
    Mx4Rows<T, D, NR> rows;
    rows.c = c;
    int lim[NR];  // last token that the lane's row may see
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int rho = rho0 + 16 * n + (lane & 15), r = min(rho, s.rows - 1);
      lim[n] = min(s.run.pos + r / a.G, s.end - 1);
      rows.start(n, (const T*)a.q + (int64_t)(s.run.row + r / a.G) * a.q_stride + (int64_t)(h * a.G + r % a.G) * D,
                 rho < s.rows, lane);
    }
    // last token that every row sees
    const int all_see = __builtin_amdgcn_readfirstlane(min(s.run.pos + rho0 / a.G, s.end - 1));
    const Mx4Places<D, P> at(lane);
    // places of a tile's halves in the pool; which of them lie in pages that are not mapped
    struct Halves {
      int64_t page[2];
      uint32_t bad;
    };
    auto halves = [&](int key) {
      Halves f;
      f.bad = 0;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        bool bad;
        f.page[t] = page_of((key + 16 * t) / P, bad) * phys_bytes;
        f.bad |= (uint32_t)bad << t;
      }
      return f;
    };
    const int last = (key_end - 1) / 32 * 32;  // (tiles begin at whole ones)
    constexpr bool ONCE = NR == 1;  // (most often the only tile of these keys)
    constexpr int kNext = 32 * kWaves;
    // The tile at `key`, and into its registers the one DEPTH tiles on as soon as they
    // are free: keys after the first product, values after the second.  (Always a tile, if need
    // be the last one again: what is on its way can be waited for in part only where
    // its number does not depend on a branch: 16 tokens at 8K to 32K 74.9 -> 62.9 us.)
    // Two tiles are under way; of fp32 rows, whose operands take the registers, one where there
    // are 32 of them (eight rows of 16 sequences at 8000 79 -> 57 us).
    constexpr int DEPTH = sizeof(T) == 4 && NR == 2 ? 1 : 2;
    Halves ahead;  // of the tile DEPTH on
    auto work = [&](Mx4Tile<D>& x, uint32_t& bad, int key) {
      const bool clean = !bad && key + 31 <= all_see;
      const int first = key + 4 * (lane >> 4);
      const Halves next = ahead;
      ahead = halves(min(key + (DEPTH + 1) * kNext, last));
      if (!clean)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          x.ve[t] = live_exponents(x.ve[t], bad >> t & 1 ? 0 : s.end - (first + 16 * t));
      rows.step(
          x,
          [&](int n, f32x4(&sc)[2]) {
            if (clean) return;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (first + 16 * t + e > lim[n] || (bad >> t & 1)) sc[t][e] = -INFINITY;
          },
          [&]() {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < 2; ++t) at.template load_keys<ONCE>(x, t, kh + next.page[t], 16 * t % P);
            __builtin_amdgcn_sched_barrier(0);
          },
          [&]() {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < 2; ++t) at.template load_values<ONCE>(x, t, vh + next.page[t], 16 * t % P);
          });
      bad = next.bad;
    };
    int key = key_begin + wave * 32;
    if (key < key_end) {
      Mx4Tile<D> x;
      uint32_t bx;
      auto load = [&](Mx4Tile<D>& z, int key) {
        const Halves f = halves(key);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          at.template load_keys<ONCE>(z, t, kh + f.page[t], 16 * t % P);
          at.template load_values<ONCE>(z, t, vh + f.page[t], 16 * t % P);
        }
        return f.bad;
      };
      bx = load(x, key);
      if constexpr (DEPTH == 2) {
        Mx4Tile<D> y;
        uint32_t by = load(y, min(key + kNext, last));
        ahead = halves(min(key + 2 * kNext, last));
        for (;;) {
          work(x, bx, key);
          if ((key += kNext) >= key_end) break;
          work(y, by, key);
          if ((key += kNext) >= key_end) break;
        }
      } else {
        ahead = halves(min(key + kNext, last));
        for (; key < key_end; key += kNext) work(x, bx, key);
      }
    }
    // results, for the join of the wavefronts
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = 16 * n + (lane & 15);
      const float l = col_sum4(rows.l[n]);
      if (lane < 16) {
        L.m[wave][r] = rows.m[n];
        L.l[wave][r] = l;
      }
      if (r < nr)
        rows.each(n, lane, [&](int d, f32x4 o) { *reinterpret_cast<f32x4*>(&L.u.o[wave][r][d]) = o; });
    }
  };

  // ---- tiles of 32 rows: this workgroup's share of the line of steps
  auto few_rows = [&]() {
    const int64_t me = kCus - 1 - blockIdx.x, mine = cut.begin(me), upto = min(cut.begin(me + 1), cut.line);
    for (int64_t pos = mine; pos < upto;) {
      int b = 0;
      int64_t local = 0, before;
      Seq s;
      find_seq(a, P, pos, L.find, tid, [&](const Seq& s) { return cut.line_of(s, a); },
               [](const Seq&) { return (int64_t)0; }, s, b, local, before);
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
        if (nr <= 16) tile_of(std::integral_constant<int, 1>{}, s, b, h, rho0, nr, key_begin, key_end);
        else tile_of(std::integral_constant<int, 2>{}, s, b, h, rho0, nr, key_begin, key_end);
        barrier();
        // a part: slot 2 k of workgroup k for what its share begins with, 2 k + 1 for what it ends with
        const bool whole = n == length;
        auto slot = [&](int64_t i) { return a.few + i * slot_floats(kRowsFew, D); };
        const __amdgpu_buffer_rsrc_t part = coherent_rsrc(slot(2 * me + (pos != mine)));
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
            const float e = __builtin_amdgcn_exp2f((L.m[w][row] - mu) * c);
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
                L.u.join, nr, parts, c, tid,
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

  // (the half of an XCD's workgroups that begins with the one way, the rest with the other)
  [[maybe_unused]] const bool turn = blockIdx.x >> 3 & 1;
  if constexpr (MANY) {
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
      if ((i == 0) != turn) {
        if (cut.many) many_rows<bf16_t, D, P>(a, cut, L, tid, wave, Mx4Stages<D, P>{L.u.many.shares}, finish);
      } else {
        if (cut.line) few_rows();
      }
    }
  } else {
    if (cut.line) few_rows();
  }
}

}  // namespace

hipError_t launch_mx4_attend(const Geometry& g, const retro_kv_cache& c, const retro_chunk& ch,
                             const void* q, int64_t q_stride, void* out, float* lse, void* ws,
                             hipStream_t s) {
  const AttendCall a = attend_call(g, c, ch, q, q_stride, out, lse, ws);
  auto go = [&](auto t, auto d, auto ps) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value, P = decltype(ps)::value;
    if constexpr (sizeof(T) == 2) {
      if (may_have_many(ch, g.batch, g.G)) {
        mx4_attend_kernel<T, D, P, true><<<kCus, kThreads, 0, s>>>(a);
        return hipGetLastError();
      }
    }
    mx4_attend_kernel<T, D, P, false><<<kCus, kThreads, 0, s>>>(a);
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
