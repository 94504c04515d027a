// Decode-step attention over the pages of the paged cache: out[h] = Softmax(z[h]) V_g over the rows that head g holds, z =
// scale <q, k>, optionally capped (cap tanh(z / cap)), biased by distance and restricted to a window of positions.
//
// The work is one line of 32-row tiles, head after head through the whole batch, cut on the device for as many workgroups as it holds at
// a time, whatever the lengths: a ragged batch, a long sequence alone and a padded one end together, and the host needs to
// know no length.  Every wavefront finds its workgroup's share by itself, with one pass over the row counts (sums over its
// lanes), in one of three cuts: units of one head where that is even; equal runs of the line, which may end in one head and go on
// in the next; whole heads by single wavefronts, for many short ones.
//
// Inside a share's part of one head the wavefronts take tiles in turn.  K goes through a wavefront's own LDS ring with
// direct-to-LDS loads, two tiles ahead, V straight into registers, one tile ahead (a lane owns the same columns of every row):
//   logits   Q x K_tile^T on the matrix cores (the G heads are the first rows of the 32-row operand, the tile's rows the columns: a
//            lane then has one row's logits for four heads, and everything up to the probabilities is four values a lane;
//            the other way round it was sixteen, three quarters of them of no head); exact products, fp32 sums
//   softmax  online, in the exp2 domain; a head's maximum is agreed on across the lanes, its sum kept per lane until the end
//   output   acc[head][columns of this lane] += p[row][head] * V[row][columns], p broadcast through LDS in fp32; V is never
//            rounded
// Pages: the numbers of a wavefront's next 64 tiles are held by its lanes, one each (two for pages of half a tile), and become
// scalars when their tile is requested, so that the table costs one trip to memory per 64 tiles, and the next head's first
// is made while this head's tiles stream.  With positions it is the next 16 tiles: four lanes each find out which rows of
// their tile are seen (tiles without any are not requested) and leave the distances in LDS for the bias.
//
// A head inside one share is finished there; otherwise each workgroup stores its part (maximum, sum, output), publishes its
// parts (two at most: of its first and its last head) at its end, and the one that finds all parts of a head published
// merges them in order.  Flags and tags are those of the decode step over the packed cache
// (xblock.h): a flag counts only if it equals the call's tag, whoever merges a head clears its flags, nobody waits.
//
// Bound by HBM: 2 * d_h * elem bytes a row.  2 x 8 heads of 131072 rows (1.07 GB) 198 us, 5.4 TB/s; 61 ragged sequences on 8 heads
// (300 MB) 71 us, 4.2 TB/s, where the workgroups' shares end within 15 us of each other (XCDs differ by a tenth in what memory
// gives them); 24 sequences with 7 heads a group, capped, biased and windowed (73 MB) 36.5 us: two trips to memory before the
// first key, 16 us of bytes, uneven windows; one sequence of 8192 rows 11 us, a chain of counts, pages, keys, parts, flags, merge.
#include <math.h>

#include "common.h"
#include "decode_parts.h"
#include "paged_common.h"
#include "tile_ring.h"
#include "xblock.h"

namespace lava {

namespace {

struct PagedArgs {
  PagedDecodeArgs p;
  float c2;                        // softmax scale * log2 e
  float2* part_ml;                 // [2 * workgroups][GP]  (maximum in log2 units, sum)
  float* part_acc;                 // [2 * workgroups][GP][D]
  unsigned long long* flags;       // [2 * workgroups]  == tag: the part is published
  unsigned long long tag;
};

// A workgroup's part of a head is stored in its first place if the head began before the workgroup's share, else in its
// second: parts 0, 1, 2, ... of a head whose first workgroup is w0.
__device__ __forceinline__ int part_slot(int w0, int u) { return u == 0 ? 2 * w0 + 1 : 2 * (w0 + u); }

// x / y rounded up, y > 0.
__device__ __forceinline__ unsigned int ceil_of(unsigned int x, unsigned int y) { return x / y + (x % y != 0u ? 1u : 0u); }
// The same for many x: inv is 1.0 / y, so the product is off by less than one.
__device__ __forceinline__ unsigned int ceil_by(unsigned int x, unsigned int y, double inv) {
  unsigned int q = (unsigned int)((double)x * inv);
  const int r = (int)(x - q * y);
  q = r < 0 ? q - 1u : r >= (int)y ? q + 1u : q;
  return q * y < x ? q + 1u : q;
}

// What a workgroup that changes heads loses, in tiles (its loads in flight drain, 6 to 9 us while the device is busy).  61 ragged sequences:
// 0 86.7 us, 3 72.2, 6 71.4, 10 74.0.
constexpr unsigned int kHeadCost = 6u;

// Tiles of a head with that many rows; -1: it cannot have them.
__device__ __forceinline__ int head_tiles(const PagedDecodeArgs& a, int rows) {
  if (rows < 0 || rows > a.max_blocks << a.page_shift) return -1;
  return (int)(((unsigned int)rows + kTileKeys - 1u) / kTileKeys);
}

// What a row's softmax sums to, in the forms that are asked for.
__device__ __forceinline__ void write_sums(const PagedDecodeArgs& p, long long row, float M, float L) {
  if (p.lse != nullptr) p.lse[row] = L == 0.0f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
  if (p.sums != nullptr) p.sums[row] = make_float2(M, L);
}

// Two values of an output row from the maximum (log2 units), the sum and the weighted values; no row seen: zeros.
template <int D>
__device__ __forceinline__ void write_row(const PagedDecodeArgs& p, int b, int g, int t, int e, float M, float L, float2 sum) {
  const long long row = (long long)b * p.H + (long long)g * p.G + t;
  const bool none = L == 0.0f;
  p.out[row * D + e] = none ? 0.0f : sum.x / L;
  p.out[row * D + e + 1] = none ? 0.0f : sum.y / L;
  if (e == 0) write_sums(p, row, M, L);
}

// The maximum, and the sum, over the 32 lanes of this lane's half of the wavefront, in each of them.
template <int CTRL>
__device__ __forceinline__ float dpp_move(float x) {
  return __uint_as_float((unsigned int)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, false));
}
template <typename F>
__device__ __forceinline__ float over_half(float x, F op) {
  x = op(x, dpp_move<0xb1>(x));                                // lane ^ 1
  x = op(x, dpp_move<0x4e>(x));                                // lane ^ 2
  x = op(x, dpp_move<0x141>(x));                               // mirrored in eight: the other four
  x = op(x, dpp_move<0x140>(x));                               // mirrored in sixteen: the other eight
  const auto h = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
__device__ __forceinline__ float max_of_half(float x) { return over_half(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float max_of_wave(float x) {
  x = max_of_half(x);
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(lane_value(__float_as_uint(fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]))), 0));
}
__device__ __forceinline__ float sum_of_half(float x) { return over_half(x, [](float a, float b) { return a + b; }); }

// The parts of one head, in order; a thread has one pair of columns, or two, and 16 loads of each kind in flight.
template <int D, int GP>
__device__ __forceinline__ void merge_parts(const PagedArgs& a, int b, int g, int w0, int parts) {
  constexpr int kPairs = GP * D / 2, kOut = (kPairs + kDecThreads - 1) / kDecThreads, kLoads = 16;
  static_assert(kPairs % kDecThreads == 0 || kPairs < kDecThreads, "threads share the pairs evenly");
  const int i = threadIdx.x;
  if (i >= kPairs) return;
  const int t = 2 * i / D, e = 2 * i % D;                      // pair o: row t + o * kRows
  constexpr int kRows = 2 * kDecThreads / D;
  float M[kOut], L[kOut];
  float2 sum[kOut];
#pragma unroll
  for (int o = 0; o < kOut; ++o) { M[o] = -INFINITY; L[o] = 0.0f; sum[o] = make_float2(0.0f, 0.0f); }
  for (int c0 = 0; c0 < parts; c0 += kLoads) {
    float2 ml[kOut][kLoads], pv[kOut][kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const bool there = c0 + u < parts;                       // uniform
      const int slot = part_slot(w0, c0 + u);
#pragma unroll
      for (int o = 0; o < kOut; ++o) {
        ml[o][u] = make_float2(-INFINITY, 0.0f);
        pv[o][u] = make_float2(0.0f, 0.0f);
        if (!there) continue;
        ml[o][u] = ld_dev_f2(&a.part_ml[slot * GP + t + o * kRows]);
        pv[o][u] = ld_dev_f2(reinterpret_cast<const float2*>(a.part_acc + (long long)slot * (GP * D) + 2 * (i + o * kDecThreads)));
      }
    }
#pragma unroll
    for (int o = 0; o < kOut; ++o) {
      float m_new = M[o];
#pragma unroll
      for (int u = 0; u < kLoads; ++u) m_new = fmaxf(m_new, ml[o][u].x);
      const float base = m_new == -INFINITY ? 0.0f : m_new;    // -inf: nothing seen so far
      const float keep = fast_exp2(M[o] - base);
      M[o] = m_new;
      L[o] *= keep;
      sum[o].x *= keep;
      sum[o].y *= keep;
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        if (c0 + u >= parts) continue;                         // uniform
        const float wgt = fast_exp2(ml[o][u].x - base);
        L[o] += wgt * ml[o][u].y;
        sum[o].x += wgt * pv[o][u].x;
        sum[o].y += wgt * pv[o][u].y;
      }
    }
  }
#pragma unroll
  for (int o = 0; o < kOut; ++o)
    if (t + o * kRows < a.p.G) write_row<D>(a.p, b, g, t + o * kRows, e, M[o], L[o], sum[o]);
}

// Wavefronts a SIMD is to hold: as many as the ring leaves room for.
template <int DT, int D>
constexpr int kWavesPerSimd = Tile<DT, D>::kRowBytes == 128 ? 3 : Tile<DT, D>::kRowBytes == 256 ? 2 : 1;

template <int DT, int D, int GP, bool OPT>
__global__ void __launch_bounds__(kDecThreads, (kWavesPerSimd<DT, D>)) paged_decode_kernel(PagedArgs a) {
  using S = DecShape<DT, D>;
  using T = Tile<DT, D>;
  constexpr int kStages = S::kStages;
  constexpr int kDpl = S::kDpl;
  __shared__ u32x4 s_tile[kDecWaves][kStages][T::kTileChunks];   // between heads: float [kDecWaves][GP][D]
  constexpr int kPs = GP < 4 ? 4 : GP;                      // floats per row in s_p (one or two 128-bit reads)
  __shared__ __attribute__((aligned(16))) float s_p[kDecWaves][kTileKeys + 1][kPs];   // probabilities; row 32: rescale factors
  __shared__ float s_m[kDecWaves][GP], s_l[kDecWaves][GP];
  constexpr int kBlock = OPT ? 16 : 64;                     // tiles whose pages a wavefront holds
  __shared__ __attribute__((aligned(16))) float s_back[OPT ? kDecWaves : 1][OPT ? 16 * kTileKeys : 4];   // distances to the rows
  __shared__ int s_flag[2], s_pend[2][3];                    // parts that wait to be published: head, first workgroup, number of parts

  const PagedDecodeArgs& p = a.p;
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int n_heads = p.batch * p.H_kv;
  const int shift = p.page_shift, page_mask = (1 << shift) - 1;

  // ---------------- this workgroup's share: sums over all heads, 64 at a time
  const bool spread = OPT && p.window > 0;
  const double inv_heads = 1.0 / (double)p.H_kv;              // h / H_kv: half a head off the border, so the product is exact enough
  constexpr int kHeld = 8;                                    // counts a lane holds at once: 512 heads in one trip to memory
  int held[kHeld];
  auto load_counts = [&](int h0) {
#pragma unroll
    for (int c = 0; c < kHeld; ++c) {
      const int h = h0 + 64 * c + lane;
      held[c] = h < n_heads ? p.head_rows[h] : 0;
    }
#pragma unroll
    for (int c = 0; c < kHeld; ++c) {
      held[c] = places_of(head_tiles(p, held[c]), spread);
      if (spread && held[c] > 0) {
        const int b = (int)(((double)(h0 + 64 * c + lane) + 0.5) * inv_heads), log_per = log_per_place(p.q_pos[b], p.window);
        held[c] = (held[c] + (1 << log_per) - 1) >> log_per;
      }
    }
  };
  unsigned int mine = 0u, full = 0u, most = 0u;
  bool empty = false;
  for (int h0 = 0; h0 < n_heads; h0 += 64 * kHeld) {
    load_counts(h0);
#pragma unroll
    for (int c = 0; c < kHeld; ++c) {
      mine += held[c] > 0 ? (unsigned int)held[c] : 0u;
      full += held[c] > 0 ? 1u : 0u;
      most = held[c] > (int)most ? (unsigned int)held[c] : most;
      empty |= h0 + 64 * c + lane < n_heads && held[c] <= 0;
    }
  }
  const unsigned int total = lane_value(wave_incl(mine), 63), n_full = lane_value(wave_incl(full), 63);
  // Heads that hold nothing, or cannot hold what their count says, are in nobody's share: workgroup h % gridDim fills in.
  if (__ballot(empty) != 0ull) {
    for (int h = blockIdx.x; h < n_heads; h += gridDim.x) {
      const int n = head_tiles(p, p.head_rows[h]);
      if (n > 0) continue;                                    // uniform
      const int b = h / p.H_kv;
      const long long row0 = (long long)b * p.H + (long long)(h - b * p.H_kv) * p.G;
      for (int i = threadIdx.x; i < p.G * D; i += kDecThreads) p.out[row0 * D + i] = n < 0 ? NAN : 0.0f;
      if ((int)threadIdx.x < p.G) write_sums(p, row0 + threadIdx.x, -INFINITY, n < 0 ? NAN : 0.0f);
    }
  }
  if (total == 0u) return;
  const float longest = max_of_wave((float)most);
  // Three ways to cut.  By heads: units of at most `share` tiles of one head, a workgroup each, if there are enough workgroups for
  // all units.  Else through the line, where a head weighs kHeadCost tiles more than it has: what it costs to change heads.
  // Parts of a long head are merged one after another, a tenth of a microsecond each, where a tile more in a share is half of
  // one: no fewer tiles in a share than the root of a quarter of the longest head's.
  const unsigned int wgs = gridDim.x, least = (unsigned int)sqrtf(0.25f * longest);
  unsigned int even = ceil_of(total, wgs), line = ceil_of(total + kHeadCost * n_full, wgs);
  if (even < least) even = least;
  if (line < least) line = least;
  // By wavefronts: each has heads of its own, and nothing is shared or merged.  For many short heads, where changing heads together costs
  // more than uneven wavefronts (rounds of tiles, half as many again allowed).  2048 heads of 40 / 300 / 900 rows 42 -> 20.5 us,
  // 93 -> 73, 196 -> 189, 1024 of 40 / 300 / 450 22.4 -> 14.2, 47 -> 41, 61 -> 56.
  const bool by_waves = 8.0f * longest * (float)ceil_of(n_full, kDecWaves * wgs) <= 3.0f * (float)line;
  unsigned int share = 0u;
  bool by_heads = false;
#pragma unroll 1
  for (int attempt = 0; attempt < 2 && !by_heads && !by_waves; ++attempt) {   // with shares as even as can be, then with those of the line
    share = ((attempt == 0 ? even : line) + 3u) & ~3u;        // a tile for every wavefront
    const double inv = 1.0 / (double)share;
    unsigned int units = 0u;
    for (int h0 = 0; h0 < n_heads; h0 += 64 * kHeld) {
      if (n_heads > 64 * kHeld) load_counts(h0);
#pragma unroll
      for (int c = 0; c < kHeld; ++c) units += held[c] > 0 ? ceil_by((unsigned int)held[c], share, inv) : 0u;
    }
    by_heads = lane_value(wave_incl(units), 63) <= wgs;       // at most one unit a head more than tiles / share: no overflow
  }
  if (!by_heads) share = line;
  const unsigned int weight = by_heads ? 0u : kHeadCost;
  // t0: this workgroup's unit, or its first place in the line
  const unsigned int t0 = by_heads ? blockIdx.x : blockIdx.x * share;
  int hb = -1;
  unsigned int head_start = 0u;                               // units, or places, before the head
  {
    const double inv = 1.0 / (double)share;
    unsigned int at = 0u;
    for (int h0 = 0; h0 < n_heads && hb < 0 && !by_waves; h0 += 64 * kHeld) {
      if (n_heads > 64 * kHeld) load_counts(h0);
#pragma unroll
      for (int c = 0; c < kHeld; ++c) {
        if (hb >= 0) continue;                                // uniform
        const unsigned int k = held[c] > 0 ? (unsigned int)held[c] : 0u;
        const unsigned int n = k == 0u ? 0u : by_heads ? ceil_by(k, share, inv) : k + weight, incl = wave_incl(n);
        const unsigned long long after = __ballot(at + incl > t0);
        if (after != 0ull) {
          const int l = __builtin_ctzll(after);
          hb = h0 + 64 * c + l;
          head_start = at + lane_value(incl, l) - lane_value(n, l);
        } else {
          at += lane_value(incl, 63);
        }
      }
    }
  }
  // The next head with rows from h on, `step` apart; n_heads: none.
  auto next_with_rows = [&](int h, int step) -> int {
    while (h < n_heads && head_tiles(p, p.head_rows[h]) <= 0) h += step;
    return h < n_heads ? h : n_heads;
  };
  const int head_step = by_waves ? kDecWaves * (int)gridDim.x : 1, stride = by_waves ? 0 : 2;   // stride: log2 of this wavefront's, in tiles
  static_assert(kDecWaves == 4, "log2");
  if (by_waves) hb = next_with_rows(wave * (int)gridDim.x + (int)blockIdx.x, head_step);
  if (hb < 0 || hb >= n_heads) return;                        // more workgroups than units, or wavefronts than heads

  using VRaw = typename RawBits<S::kBpl>::type;
  TileDma<DT, D> dma;
  dma.init(lane);
  u32x4* ring = s_tile[wave][0];
  FragReader<DT, D> frags;
  frags.init_at(lane, lds_addr(ring));
  const unsigned int p_addr = lds_addr(&s_p[wave][0][0]);
  const int col = lane & 31, half = lane >> 5;
  const unsigned int p_mine = p_addr + (unsigned int)((col * kPs + (GP > 4 ? 4 * half : 0)) * 4);   // this row, this lane's four heads
  const unsigned int p_alpha = p_addr + (unsigned int)((kTileKeys * kPs + (GP > 4 ? 4 * half : 0)) * 4);
  const unsigned int v_lane = (unsigned int)lane * S::kBpl;   // a row is a uniform address plus this
  const float inv_cap = p.cap > 0.0f ? 1.0f / p.cap : 0.0f;
  const unsigned int window = p.window > 0 ? (unsigned int)p.window : 0x80000000u;

  // Pages of tile0, tile0 + 2^stride, ... of head h, kBlock of them, as far as there are `here`: a lane each, or four (OPT)
  auto load_pages = [&](int h, int rows_h, int columns, int tile0, int here, int& page_a, int& page_b) {
    const int i = OPT ? lane >> 2 : lane;
    const unsigned int row0 = row_at(tile0 + (i << stride), columns);
    const int* table = p.block_table + (long long)h * p.max_blocks;
    page_a = page_b = 0;
    if (i < here && (!OPT || row0 < (unsigned int)rows_h)) {
      page_a = table[row0 >> shift];
      page_b = shift == 4 && row0 + 16u < (unsigned int)rows_h ? table[(row0 >> 4) + 1u] : page_a;
    }
  };

  if (threadIdx.x < 2) s_pend[threadIdx.x][2] = 0;             // of the first and of the last head of the share
  struct HeadOrder {
    int rows, columns, order, log_per, tiles;                 // columns of its tiles' order, tiles in that order, log2 of how many make a place, places
  };
  auto head_order = [&](int h) -> HeadOrder {
    HeadOrder o;
    o.rows = p.head_rows[h];
    const int n = head_tiles(p, o.rows);
    o.columns = spread_columns(n, spread);
    o.order = places_of(n, spread);
    o.log_per = spread ? log_per_place(p.q_pos[h / p.H_kv], p.window) : 0;
    o.tiles = (o.order + (1 << o.log_per) - 1) >> o.log_per;
    return o;
  };
  int page_a, page_b;
  bool pages_ready = false;
  // In the line a head's tiles follow its weight: tile j is place head_start + weight + j.
  const unsigned int t1 = t0 + share, line_end = total + weight * n_full;
  unsigned int done = 0u;                                     // tiles of the share so far
  for (;;) {
    const int b = hb / p.H_kv, g = hb - b * p.H_kv;
    const HeadOrder of = head_order(hb);
    const int rows = of.rows, columns = of.columns, order = of.order, log_per = of.log_per, tiles = of.tiles;
    const unsigned int at = head_start + weight;              // place of the head's first tile
    int ta, tb;                                               // its places that are this share's
    if (by_waves) {
      ta = 0;
      tb = tiles;
    } else if (by_heads) {
      ta = (int)((t0 - head_start) * share);
      tb = tiles - ta < (int)share ? tiles : ta + (int)share;
    } else {
      ta = t0 > at ? (int)(t0 - at) : 0;
      tb = t1 <= at ? 0 : t1 - at < (unsigned int)tiles ? (int)(t1 - at) : tiles;
    }
    if (ta >= tb) return;                                     // the share ends inside the first head's weight
    bool last = by_heads || (!by_waves && (at + (unsigned int)tiles + weight >= t1 || at + (unsigned int)tiles >= line_end));
    const int q_pos = OPT && p.pos != nullptr ? p.q_pos[b] : 0;
    // wavefronts take turns through the whole share, so that each has as many tiles as the others
    const int pa = ta << log_per, pb = tb == tiles ? order : tb << log_per;   // in the order of the head's tiles
    const int first = by_waves ? 0 : pa + (int)(((unsigned int)wave - done) & (kDecWaves - 1));
    const int cnt = first < pb ? (pb - first + (1 << stride) - 1) >> stride : 0;   // this wavefront's tiles
    if (!pages_ready) load_pages(hb, rows, columns, first, cnt < kBlock ? cnt : kBlock, page_a, page_b);

    // the group's query rows as the 32-row operand: row t < G is head g * G + t
    u32x4 qf[T::kSteps];
#pragma unroll
    for (int j = 0; j < T::kSteps; ++j) {
      u32x4 x = u32x4{0u, 0u, 0u, 0u};
      if (col < p.G) x = reinterpret_cast<const u32x4*>(p.q)[((long long)b * p.H + (long long)g * p.G + col) * T::kCpr + 2 * j + half];
      qf[j] = x;
    }
    // of heads 4 * half + v of the group; the sums are those of this lane's rows
    float slope[4], m_run[4], l_run[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      slope[v] = OPT && p.slopes != nullptr && 4 * half + v < p.G ? p.slopes[g * p.G + 4 * half + v] * kLog2e : 0.0f;
      m_run[v] = -INFINITY;
      l_run[v] = 0.0f;
    }
    float acc[GP][kDpl];
#pragma unroll
    for (int i = 0; i < GP; ++i)
#pragma unroll
      for (int e = 0; e < kDpl; ++e) acc[i][e] = 0.0f;

    int next_head = hb, next_a = 0, next_b = 0;
    for (int i0 = 0; i0 == 0 || i0 < cnt; i0 += kBlock) {
      const int tile0 = first + (i0 << stride);
      const int here = cnt - i0 < kBlock ? cnt - i0 : kBlock;
      if (i0 > 0) load_pages(hb, rows, columns, tile0, here, page_a, page_b);
      unsigned int seen = 0xffffffffu;                        // rows of the lane's tile that count (OPT)
      {
        const bool bad = page_a < 0 || page_a >= p.n_pages || page_b < 0 || page_b >= p.n_pages;
        if (__ballot(bad) != 0ull) {                          // the head's result is NaN: any page will do
#pragma unroll
          for (int v = 0; v < 4; ++v) l_run[v] = NAN;
          if (bad) page_a = page_b = 0;
        }
        if (OPT) {
          const int i = lane >> 2, part = lane & 3;           // rows 8 part .. 8 part + 7 of tile i
          const unsigned int row0 = row_at(tile0 + (i << stride), columns);
          seen = 0u;
          if (i < here && row0 < (unsigned int)rows) {
            int4 x = make_int4(q_pos, q_pos, q_pos, q_pos), x2 = x;
            if (p.pos != nullptr) {                            // uniform
              const long long place = shift == 4 ? ((long long)(part < 2 ? page_a : page_b) << 4) + 8 * (part & 1)
                                                 : ((long long)page_a << shift) + ((int)row0 & page_mask) + 8 * part;
              x = *reinterpret_cast<const int4*>(p.pos + place);
              x2 = *reinterpret_cast<const int4*>(p.pos + place + 4);
            }
            const int y[8] = {x.x, x.y, x.z, x.w, x2.x, x2.y, x2.z, x2.w};
            float back[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const unsigned int d = (unsigned int)q_pos - (unsigned int)y[e];   // a later row: 2^31 and more
              back[e] = (float)d;
              if (d < window && (int)row0 + 8 * part + e < rows) seen |= 1u << e;
            }
            float* dst = &s_back[wave][lane * 8];
#pragma unroll
            for (int e = 0; e < 8; ++e) dst[e] = back[e];
          }
          seen <<= 8 * part;
          seen |= (unsigned int)__shfl_xor((int)seen, 1);
          seen |= (unsigned int)__shfl_xor((int)seen, 2);
        }
      }
      unsigned long long todo = OPT ? __ballot(seen != 0u) & 0x1111111111111111ull : here == 64 ? ~0ull : (1ull << here) - 1ull;
      auto row_of = [&](int j) -> int { return (int)row_at(tile0 + ((OPT ? j >> 2 : j) << stride), OPT ? columns : 0); };   // first row of lane j's tile, which the head has
      // place in the pool of the first rows of the tile's two halves
      auto half_a = [&](int j) -> long long {
        return ((long long)(int)lane_value((unsigned int)page_a, j) << shift) + (row_of(j) & page_mask);
      };
      auto half_b = [&](int j, long long at) -> long long {
        return shift == 4 ? (long long)(int)lane_value((unsigned int)page_b, j) << 4 : at + 16;
      };
      auto next_tile = [&]() -> int {                          // -1: none left
        if (todo == 0ull) return -1;
        const int j = __builtin_ctzll(todo);
        todo &= todo - 1ull;
        return j;
      };
      auto issue_k = [&](int j, int stage) {                   // rows behind the head's last one come along, unused
        const long long at = half_a(j), bt = half_b(j, at);
        const char* ka = p.k + at * T::kRowBytes;
        const char* kb = p.k + bt * T::kRowBytes - T::kTileBytes / 2;
        dma.issue_halves(ka, kb, ring + stage * T::kTileChunks);
      };
      auto load_v = [&](VRaw (&dst)[kTileKeys], int j) {
        const long long at = half_a(j), bt = half_b(j, at);
        const char* va = p.v + at * T::kRowBytes;
        const char* vb = p.v + bt * T::kRowBytes - T::kTileBytes / 2;
#pragma unroll
        for (int kk = 0; kk < kTileKeys; ++kk)
          dst[kk] = *reinterpret_cast<const VRaw*>((kk < kTileKeys / 2 ? va : vb) + kk * T::kRowBytes + v_lane);
      };

      // Vector-memory operations complete in issue order and the K ring is awaited by count, so the order below is part of the
      // protocol:  K_0, K_1 | V_0 | then per tile i:  K_{i+2}, V_{i+1}  (other loads among them only make a wait longer)
      int j0 = next_tile(), j1 = next_tile(), j2 = next_tile();   // current tile, the next, the one after
      if (j0 >= 0) issue_k(j0, 0);
      if (j1 >= 0) issue_k(j1, 1);
      asm volatile("" ::: "memory");
      VRaw v0[kTileKeys], v1[kTileKeys];
      if (j0 >= 0) load_v(v0, j0);
      if (i0 == 0 && !last) {                                  // the next head of the share, while this one streams
        next_head = next_with_rows(hb + head_step, head_step);
        last = next_head >= n_heads;                           // by wavefronts; in the line there is one
      }
      if (i0 == 0 && !last) {
        const HeadOrder next = head_order(next_head);
        const unsigned int n_at = at + (unsigned int)tiles + weight;
        const int n_tb = !by_waves && t1 - n_at < (unsigned int)next.tiles ? (int)(t1 - n_at) << next.log_per : next.order;
        const int n_first = by_waves ? 0 : (int)(((unsigned int)wave - done - (unsigned int)(pb - pa)) & (kDecWaves - 1));
        const int n_cnt = n_first < n_tb ? (n_tb - n_first + (1 << stride) - 1) >> stride : 0;
        load_pages(next_head, next.rows, next.columns, n_first, n_cnt < kBlock ? n_cnt : kBlock, next_a, next_b);
      }

      auto step = [&](auto par, VRaw (&v_cur)[kTileKeys], VRaw (&v_next)[kTileKeys]) {
        constexpr int PAR = decltype(par)::value;              // ring stage of the current tile
        const int left = rows - row_of(j0);                    // rows from this tile on
        const unsigned int mask = OPT ? lane_value(seen, j0) : left >= kTileKeys ? ~0u : (1u << left) - 1u;   // rows that count
        {
          // everything older than this tile's V (32 loads) and, if it was requested, the next K has landed
          if (j1 >= 0) wait_vmcnt<T::kLoads + kTileKeys>(); else wait_vmcnt<kTileKeys>();
          u32x4 kf[T::kSteps];
          frags.template read_at<PAR * T::kTileBytes>(kf);     // in registers on return: the stage is free
          if (j2 >= 0) issue_k(j2, PAR);
          asm volatile("" ::: "memory");
          f32x16 sum = {0}, sum2 = {0};                        // two chains halve the latency of dependent products
#pragma unroll
          for (int j = 0; j < T::kSteps; j += 2) {
            sum = mfma_chunk<DT>(qf[j], kf[j], sum);
            sum2 = mfma_chunk<DT>(qf[j + 1], kf[j + 1], sum2);
          }
          float x[4];                                          // row `col` of the tile, heads 4 * half + v
#pragma unroll
          for (int v = 0; v < 4; ++v) x[v] = sum[v] + sum2[v];
          if (OPT && p.cap > 0.0f) {                           // uniform
#pragma unroll
            for (int v = 0; v < 4; ++v) x[v] = capped(x[v] * p.scale, p.cap, inv_cap) * kLog2e;
          } else {
#pragma unroll
            for (int v = 0; v < 4; ++v) x[v] *= a.c2;
          }
          if (OPT) {
            if (p.slopes != nullptr) {                         // uniform
              const float back = lds_read32(lds_addr(&s_back[wave][0]) + (unsigned int)(((j0 >> 2) * kTileKeys + col) * 4));
#pragma unroll
              for (int v = 0; v < 4; ++v) x[v] -= slope[v] * back;
            }
          }
          if (mask != ~0u) {                                   // uniform; whatever the other rows hold
            const bool on = (mask >> col) & 1u;
#pragma unroll
            for (int v = 0; v < 4; ++v) x[v] = on ? x[v] : -INFINITY;
          }
          float e[4], alpha[4];
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const float m_new = fmaxf(m_run[v], max_of_half(x[v]));
            const float base = m_new == -INFINITY ? 0.0f : m_new;   // logits that are all -inf
            alpha[v] = fast_exp2(m_run[v] - base);
            e[v] = fast_exp2(x[v] - base);
            l_run[v] = l_run[v] * alpha[v] + e[v];
            m_run[v] = m_new;
          }
          if (GP > 4 || half == 0) {
            lds_write128(p_mine, e);
            if (col == 0) lds_write128(p_alpha, alpha);
          }
        }
        lds_reads_done();                                      // LDS operations of a wavefront execute in order
        {
          if (j1 >= 0) load_v(v_next, j1);
          asm volatile("" ::: "memory");
          if (mask != ~0u) {
#pragma unroll
            for (int kk = 0; kk < kTileKeys; ++kk) v_cur[kk] = (mask >> kk) & 1u ? v_cur[kk] : VRaw{};
          }
          u32x4 al[kPs / 4];
          static_for<kPs / 4>([&](auto cc) {
            constexpr int c = decltype(cc)::value;
            lds_read128_at<(kTileKeys * kPs + 4 * c) * 4>(p_addr, al[c]);
          });
#pragma unroll
          for (int i = 0; i < GP; ++i)
#pragma unroll
            for (int e = 0; e < kDpl; ++e) acc[i][e] *= __uint_as_float(al[i / 4][i % 4]);
          // probabilities of four rows per read batch
          static_for<kTileKeys / 4>([&](auto kc) {
            constexpr int k4 = 4 * decltype(kc)::value;
            u32x4 pr[kPs / 4][4];
            static_for<kPs / 4>([&](auto cc) {
              constexpr int c = decltype(cc)::value;
              lds_read128x4_strided<kPs * 4, (k4 * kPs + 4 * c) * 4>(p_addr, pr[c][0], pr[c][1], pr[c][2], pr[c][3]);
            });
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              float vx[kDpl];
              unpack_v<DT, D>(v_cur[k4 + kk], vx);
#pragma unroll
              for (int i = 0; i < GP; ++i) {
                const float pw = __uint_as_float(pr[i / 4][kk][i % 4]);
#pragma unroll
                for (int e = 0; e < kDpl; ++e) acc[i][e] = fmaf(pw, vx[e], acc[i][e]);
              }
            }
            // pin the accumulators here: otherwise the multiply-adds of all batches sink below the reads of all batches, which
            // then have to stay in registers together
#pragma unroll
            for (int i = 0; i < GP; ++i)
#pragma unroll
              for (int e = 0; e < kDpl; ++e) asm volatile("" : "+v"(acc[i][e]));
          });
        }
        j0 = j1;
        j1 = j2;
        j2 = next_tile();
      };
      while (j0 >= 0) {
        step(std::integral_constant<int, 0>{}, v0, v1);
        if (j0 < 0) break;
        step(std::integral_constant<int, 1>{}, v1, v0);
      }
      wait_vmcnt<0>();
    }

    if (by_waves) {
      // ---------------- the head is this wavefront's alone
#pragma unroll
      for (int v = 0; v < 4; ++v) l_run[v] = sum_of_half(l_run[v]);
#pragma unroll
      for (int i = 0; i < GP; ++i) {
        if (i >= p.G) continue;                               // uniform
        const float M = __uint_as_float(lane_value(__float_as_uint(m_run[i & 3]), i < 4 ? 0 : 32));
        const float L = __uint_as_float(lane_value(__float_as_uint(l_run[i & 3]), i < 4 ? 0 : 32));
        const long long row = (long long)b * p.H + (long long)g * p.G + i;
#pragma unroll
        for (int e = 0; e < kDpl; ++e) p.out[row * D + lane * kDpl + e] = L == 0.0f ? 0.0f : acc[i][e] / L;
        if (lane == 0) write_sums(p, row, M, L);
      }
      if (last) return;
      hb = next_head;
      page_a = next_a;
      page_b = next_b;
      pages_ready = true;
      continue;
    }
    // ---------------- merge the wavefronts
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      l_run[v] = sum_of_half(l_run[v]);
      if (col == 0 && 4 * half + v < GP) {
        s_m[wave][4 * half + v] = m_run[v];
        s_l[wave][4 * half + v] = l_run[v];
      }
    }
    __syncthreads();                                          // every wavefront is done with its ring
    float (*s_acc)[GP][D] = reinterpret_cast<float (*)[GP][D]>(&s_tile[0][0][0]);
#pragma unroll
    for (int i = 0; i < GP; ++i)
#pragma unroll
      for (int e = 0; e < kDpl; ++e) s_acc[wave][i][lane * kDpl + e] = acc[i][e];
    __syncthreads();
    const bool whole = ta == 0 && tb == tiles;
    const int slot = 2 * (int)blockIdx.x + (ta > 0 ? 0 : 1);
    constexpr int kPairs = GP * D / 2;
#pragma unroll
    for (int j = 0; j < (kPairs + kDecThreads - 1) / kDecThreads; ++j) {
      const int idx = 2 * ((int)threadIdx.x + kDecThreads * j), i = idx / D, e = idx % D;
      if (i >= GP) continue;
      float M = s_m[0][i];
#pragma unroll
      for (int w2 = 1; w2 < kDecWaves; ++w2) M = fmaxf(M, s_m[w2][i]);
      const float base = M == -INFINITY ? 0.0f : M;
      float L = 0.0f;
      float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int w2 = 0; w2 < kDecWaves; ++w2) {
        const float wgt = fast_exp2(s_m[w2][i] - base);
        L += wgt * s_l[w2][i];
        sum.x += wgt * s_acc[w2][i][e];
        sum.y += wgt * s_acc[w2][i][e + 1];
      }
      if (!whole) {
        st_dev_f2(reinterpret_cast<float2*>(a.part_acc + (long long)slot * (GP * D) + idx), sum.x, sum.y);
        if (e == 0) st_dev_f2(&a.part_ml[slot * GP + i], M, L);
      } else if (i < p.G) {
        write_row<D>(p, b, g, i, e, M, L, sum);
      }
    }
    if (!whole) {
      const int w0 = (int)(by_heads ? head_start : at / share);
      const int parts = by_heads ? (int)ceil_of((unsigned int)tiles, share) : (int)((at + (unsigned int)tiles - 1u) / share) - w0 + 1;
      if (threadIdx.x == 0) {
        int* pend = s_pend[ta > 0 ? 0 : 1];
        pend[0] = hb;
        pend[1] = w0;
        pend[2] = parts;
      }
    }
    if (last) break;
    __syncthreads();                                          // the ring and s_m are free again
    head_start = at + (unsigned int)tiles;
    done += (unsigned int)(pb - pa);
    hb = next_head;
    page_a = next_a;
    page_b = next_b;
    pages_ready = true;
  }

  // ---------------- publish the parts; merge every head all of whose parts are published
  drain_vmem();
  __syncthreads();                                            // every thread's share of the parts is visible to the device
  if (s_pend[0][2] == 0 && s_pend[1][2] == 0) return;         // uniform
  if (wave == 0) {
    if (lane < 2 && s_pend[lane][2] > 0) {
      st_dev(&a.flags[2 * blockIdx.x + lane], a.tag);
      drain_vmem();
    }
    for (int i = 0; i < 2; ++i) {
      const int w0 = s_pend[i][1], parts = s_pend[i][2];
      bool all = parts > 0;
      for (int u = lane; u < parts; u += 64) all &= ld_dev(&a.flags[part_slot(w0, u)]) == a.tag;
      const bool every = __ballot(!all) == 0ull;
      if (lane == 0) s_flag[i] = every ? 1 : 0;
    }
  }
  __syncthreads();
#pragma unroll 1
  for (int i = 0; i < 2; ++i) {
    if (s_flag[i] == 0) continue;
    const int h = (int)lane_value((unsigned int)s_pend[i][0], 0), w0 = (int)lane_value((unsigned int)s_pend[i][1], 0),
              parts = (int)lane_value((unsigned int)s_pend[i][2], 0);
    for (int u = threadIdx.x; u < parts; u += kDecThreads) st_dev(&a.flags[part_slot(w0, u)], 0ull);
    const int b = h / p.H_kv;
    merge_parts<D, GP>(a, b, h - b * p.H_kv, w0, parts);
  }
}

// Workgroups of a launch: what the device holds at a time, at most four a compute unit.
constexpr int kMostPerCu = 4;
template <typename K>
int resident(K kernel) {
  int per = 0;
  if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, kDecThreads, 0) != hipSuccess || per < 1) {
    discard_stale_error();
    per = 1;
  }
  return (per < kMostPerCu ? per : kMostPerCu) * device_cus();
}

struct PagedLayout {
  size_t off_ml, off_acc, off_flags, bytes;
};
PagedLayout make_layout(const lava_layer_desc& d) {
  PagedLayout l;
  const size_t slots = 2 * (size_t)kMostPerCu * device_cus(), gp = padded_group(d.n_q_heads / d.n_kv_heads);
  l.off_ml = 0;
  l.off_acc = align_up(slots * gp * sizeof(float2));
  l.off_flags = l.off_acc + align_up(slots * gp * d.head_dim * sizeof(float));
  l.bytes = l.off_flags + align_up(slots * sizeof(unsigned long long));
  return l;
}

template <int DT, int D, int GP, bool OPT>
int32_t launch_one(const PagedArgs& a, hipStream_t s) {
  static const int wgs = resident(paged_decode_kernel<DT, D, GP, OPT>);
  ProfScope ps(KID_PAGED_DECODE, s);
  hipLaunchKernelGGL((paged_decode_kernel<DT, D, GP, OPT>), dim3((unsigned)wgs), dim3(kDecThreads), 0, s, a);
  return launch_status();
}

}  // namespace

size_t paged_decode_bytes(const lava_layer_desc& d) { return make_layout(d).bytes; }

int32_t launch_paged_decode(const lava_layer_desc& d, const PagedDecodeArgs& p, void* ws, hipStream_t s) {
  PagedArgs a;
  a.p = p;
  a.c2 = p.scale * kLog2e;
  const PagedLayout l = make_layout(d);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + l.off_ml);
  a.part_acc = reinterpret_cast<float*>(static_cast<char*>(ws) + l.off_acc);
  a.flags = reinterpret_cast<unsigned long long*>(static_cast<char*>(ws) + l.off_flags);
  a.tag = next_tag();
  const int gp = padded_group(p.G);
  const bool options = p.pos != nullptr || p.cap > 0.0f;
#define LAVA_PAGED_CASE(DT, D, GP) \
  if (d.dtype == DT && d.head_dim == D && gp == GP)        \
    return options ? launch_one<DT, D, GP, true>(a, s) : launch_one<DT, D, GP, false>(a, s);
#define LAVA_PAGED_GROUPS(DT, D) LAVA_PAGED_CASE(DT, D, 1) LAVA_PAGED_CASE(DT, D, 2) LAVA_PAGED_CASE(DT, D, 4) LAVA_PAGED_CASE(DT, D, 8)
  LAVA_PAGED_GROUPS(LAVA_BF16, 128)
  LAVA_PAGED_GROUPS(LAVA_BF16, 64)
  LAVA_PAGED_GROUPS(LAVA_F32, 128)
  LAVA_PAGED_GROUPS(LAVA_F32, 64)
#undef LAVA_PAGED_GROUPS
#undef LAVA_PAGED_CASE
  return LAVA_ERR_SHAPE;
}

}  // namespace lava
