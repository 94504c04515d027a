// Decode-step attention of groups of sequences that share pages: softmax over a head's rows splits into the rows of the pages that
// a group has in common and a sequence's own,
//   out = (e^(m_c) a_c + e^(m_o) a_o) / (e^(m_c) l_c + e^(m_o) l_o),   m, l, a: maximum, sum and weighted values of either,
// and the common part of all n sequences of a group with G query heads a KV head is one matrix product of n * G queries.
//
//   plan    a workgroup per group and head: leading blocks that the tables of all its sequences have in common; what is left; the list
//           of items: up to 256 / G sequences of a group, one head
//   rows    the items' rows, cut into equal units of stages (64 KiB of keys and values) for as many workgroups as the device holds; then,
//           of up to kOwnHeads heads, what is left of each, whose queries are the G of one sequence, by whoever is done
//   own     of more heads: the decode step over pages, over tables of what is left
//   merge   the parts of the common rows and the own ones, per sequence and head
//
// Rows: a workgroup of eight wavefronts.  A stage's keys and values come to LDS by direct-to-LDS loads, one stage ahead (in a
// window only stages that hold a row of it).  A wavefront has 32 queries as the columns of its products and takes every n-th tile of
// 32 rows, n = 8 / tiles of queries:
//   logits  K_tile x Q^T: a lane has 16 of a query's 32 logits
//   softmax online, in the exp2 domain; the other 16 are in lane ^ 32
//   output  V_tile^T x P^T: in the order in which the first product leaves the rows to a lane they are the operand of the second, so
//           probabilities stay in registers.  bf16: V is read transposed from LDS, a probability is three bf16 parts (8 + 8 +
//           8 bits), so that products are exact and sums 32 bits, as in the decode step over pages (with two parts an output
//           would be off by 2.4e-6 of itself)
// Rows that are masked may hold anything there.  A product cannot leave them out, so a sequence's head whose sums are not all
// finite is marked, and merge computes its outputs again, row by row.  (A query is a column of the products: one that is no number
// leaves the others of its item as they are.)
//
// Bound by HBM for few queries: 4 groups of 4 sequences with 8 KV heads of 65536 rows (1.07 GB) 208 us a step, 5.2 TB/s.  For many by
// products and the softmax between them in turn: 64 sequences over 8 heads of 131072 rows need 275 GFLOP with the three parts; rows 287 us
// (by events, own rows among them), 0.96 PFLOP/s with the matrix cores busy for 45 % at 1.95 GHz, where a large product of the library has
// 1.1 to 1.3 with 66 % at 1.5 to 1.7.  Plan 16, merge 13, the step 309.  Six groups of 3 to 17 sequences, 7 heads each, capped, biased and in
// windows of 8192 of up to 65536 positions: rows 66 us, of which cap and bias take 6; neither bytes (1.3 TB/s) nor products (8 % busy),
// but units that begin unhidden and hold unevenly many stages of the window.  32 bits: by the 32-bit matrix instructions, which two or four
// of the eight wavefronts of few queries issue.
#include <math.h>

#include "common.h"
#include "decode_parts.h"
#include "paged_common.h"
#include "tile_ring.h"

namespace lava {

namespace {

constexpr int kShWaves = 8, kShThreads = kShWaves * 64;
constexpr int kShRows = 32 * kShWaves;         // query rows of an item at most
constexpr int kStageBytes = 65536;             // keys and values

struct SharedItem {
  int first_seq, n_seq, head, rows;            // rows in common
  int lead, skip;                              // a sequence that holds them, its blocks before them
};
struct SharedParts {
  int row, units;                              // first row of its parts, number of parts (each n_seq * G rows)
};

struct SharedArgs {
  PagedDecodeArgs p;                           // over the whole tables
  int n_groups;
  const int32_t* group_start;
  float c2;
  int own_here;                                // own rows are units too; else the decode step over pages has them
  int own_base;                                // first row of the parts of own rows
  int* n_items;                                // number of items; units that were taken out of turn
  SharedItem* items;
  SharedParts *parts, *own_parts;              // [items], [batch][H_kv]
  int *marked, *head_marked;                   // [items] 2: a page is not in the pool; [batch][H_kv] 1: sums that are not finite, 2: of own rows, a page
  int* item_of;                                // [batch][H_kv] item that has the sequence's common rows, -1: none
  int *rest_rows, *skip;                       // [batch][H_kv] rows that are left (as a unit's: -1 if there cannot be as many), blocks in common
  int* rest_table;                             // [batch][H_kv][max_blocks] where own rows are decoded by themselves
  float2* rest_sums;                           // [batch][H] and what they sum to
  float2* part_ml;                             // [rows] maximum (log2 units) and sum
  float* part_acc;                             // [rows][D]
};

// ---------------------------------------------------------------- plan
constexpr int kPlanShThreads = 1024, kPlanShWaves = kPlanShThreads / 64;
__global__ void __launch_bounds__(kPlanShThreads) shared_plan_kernel(const SharedArgs a) {
  __shared__ int s_bad, s_blocks[kPlanShWaves], s_before[kPlanShWaves], s_all[kPlanShWaves], s_lead[kPlanShWaves], s_some[kPlanShWaves];
  const PagedDecodeArgs& p = a.p;
  const int group = blockIdx.x / p.H_kv, g = blockIdx.x - group * p.H_kv, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int seqs = kShRows / p.G, P = 1 << p.page_shift;
  const int from = a.group_start[group], to = a.group_start[group + 1];   // on their way while the others are looked at
  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();
  int before = 0, all = 0;                                     // blocks of sequences of the groups before, of all
  for (int i = threadIdx.x; i < a.n_groups; i += kPlanShThreads) {
    const int x = a.group_start[i], y = a.group_start[i + 1];
    if (x < 0 || y < x || y > p.batch || (i == 0 && x != 0) || (i == a.n_groups - 1 && y != p.batch)) {
      s_bad = 1;
    } else {
      const int n = (y - x + seqs - 1) / seqs;
      before += i < group ? n : 0;
      all += n;
    }
  }
  before = (int)lane_value(wave_incl((unsigned int)before), 63);
  all = (int)lane_value(wave_incl((unsigned int)all), 63);
  if (lane == 0) {
    s_before[wave] = before;
    s_all[wave] = all;
  }
  __syncthreads();
  const bool bad = s_bad != 0;
  before = all = 0;
  for (int w = 0; w < kPlanShWaves; ++w) {
    before += s_before[w];
    all += s_all[w];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.n_items[0] = bad ? 0 : all * p.H_kv;
    a.n_items[1] = 0;
  }
  // groups that are none: every sequence by itself
  const int b0 = bad ? group : from, b1 = bad ? p.batch : to, step = bad ? a.n_groups : 1;
  int common = 0, lead = 0x7fffffff;
  if (!bad && b1 - b0 > 1) {                                   // uniform
    auto held = [&](int b) { return p.head_rows[(long long)b * p.H_kv + g]; };
    auto table = [&](int b) { return p.block_table + ((long long)b * p.H_kv + g) * p.max_blocks; };
    // the sequence to compare with, full blocks that all have
    int least = 0x7fffffff, some = 0;
    for (int b = b0 + threadIdx.x; b < b1; b += kPlanShThreads) {
      const int rows = held(b);
      if (rows == 0) continue;
      const int blocks = rows < 0 || rows > p.max_blocks << p.page_shift ? 0 : rows >> p.page_shift;
      least = blocks < least ? blocks : least;
      lead = b < lead ? b : lead;
      ++some;
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      least = min(least, __shfl_xor(least, m));
      lead = min(lead, __shfl_xor(lead, m));
      some += __shfl_xor(some, m);
    }
    if (lane == 0) {
      s_blocks[wave] = least;
      s_lead[wave] = lead;
      s_some[wave] = some;
    }
    __syncthreads();
    some = 0;
    for (int w = 0; w < kPlanShWaves; ++w) {
      least = min(least, s_blocks[w]);
      lead = min(lead, s_lead[w]);
      some += s_some[w];
    }
    if (some > 1) {
      // a wavefront 64 blocks: the first one in which a sequence differs, kCompared of them at a time
      constexpr int kCompared = 32;
      const int* first = table(lead);
      common = least;
      for (int j0 = 64 * wave; j0 < least; j0 += 64 * kPlanShWaves) {
        const int j = j0 + lane < least ? j0 + lane : least - 1, x = first[j];
        bool differs = false;
        for (int c1 = b0; c1 < b1; c1 += 64) {
          const unsigned long long there = __ballot(c1 + lane < b1 && held(c1 + lane < b1 ? c1 + lane : b0) != 0);
          for (int c0 = 0; c0 < 64 && (there >> c0) != 0ull; c0 += kCompared) {
            int y[kCompared];
#pragma unroll
            for (int i = 0; i < kCompared; ++i) y[i] = table((there >> (c0 + i)) & 1ull ? c1 + c0 + i : lead)[j];
#pragma unroll
            for (int i = 0; i < kCompared; ++i) differs |= y[i] != x;
          }
        }
        const unsigned long long off = __ballot(differs);
        if (off != 0ull) {
          const int at = j0 + __builtin_ctzll(off);
          common = at < common ? at : common;
          break;
        }
      }
    }
    __syncthreads();                                           // s_blocks is read
    if (lane == 0) s_blocks[wave] = common;
    __syncthreads();
    for (int w = 0; w < kPlanShWaves; ++w) common = min(common, s_blocks[w]);
  }
  const int n = b1 - b0, blocks = bad ? 0 : (n + seqs - 1) / seqs, item0 = before * p.H_kv + g * blocks;
  for (int i = threadIdx.x; i < blocks; i += kPlanShThreads) {
    SharedItem it;
    it.first_seq = b0 + i * seqs;
    it.n_seq = n - i * seqs < seqs ? n - i * seqs : seqs;
    it.head = g;
    it.rows = common << p.page_shift;
    it.lead = common > 0 ? lead : b0;
    it.skip = 0;
    a.items[item0 + i] = it;
    a.marked[item0 + i] = 0;
  }
  // what is left: a wavefront four sequences at a time
  for (int c0 = b0 + wave * step; c0 < b1; c0 += 4 * kPlanShWaves * step) {
    long long h[4];
    int rows[4], skip[4], left[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = c0 + i * kPlanShWaves * step;
      h[i] = (long long)(b < b1 ? b : c0) * p.H_kv + g;
      rows[i] = p.head_rows[h[i]];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool there = c0 + i * kPlanShWaves * step < b1;
      skip[i] = rows[i] == 0 ? 0 : common;
      left[i] = a.own_here != 0 || !there || rows[i] <= 0 || rows[i] > p.max_blocks << p.page_shift ? 0 : ((rows[i] + P - 1) >> p.page_shift) - skip[i];
      y[i] = lane < left[i] ? p.block_table[h[i] * p.max_blocks + skip[i] + lane] : 0;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = c0 + i * kPlanShWaves * step;
      if (b >= b1) continue;
      if (lane == 0) {
        const bool none = rows[i] < 0 || rows[i] > p.max_blocks << p.page_shift;
        a.rest_rows[h[i]] = a.own_here != 0 && none ? -1 : rows[i] - (skip[i] << p.page_shift);
        a.skip[h[i]] = skip[i];
        a.head_marked[h[i]] = 0;
        a.item_of[h[i]] = skip[i] > 0 ? item0 + (b - b0) / seqs : -1;
      }
      int* rest = a.rest_table + h[i] * p.max_blocks;
      if (lane < left[i]) rest[lane] = y[i];
      for (int j = 64 + lane; j < left[i]; j += 64) rest[j] = p.block_table[h[i] * p.max_blocks + skip[i] + j];
    }
  }
}

// ---------------------------------------------------------------- rows
// A probability is relative to a maximum that moves only when a logit exceeds it by more than this (in log2 units): sums grow by 2^8 at
// most, and half of the tiles need no rescaling of the output (296 -> 283 us).
constexpr float kSlack = 8.0f;

// (sequence, head) pairs whose own rows are units of the same launch, at most; more are many small units, and their number is found again by
// every workgroup.  Groups x sequences over 16384 rows and 300 own ones, bf16, 8 KV heads, us a step with own rows apart and here:
//   256 heads   4 x 8 85.5 and 79.7, 1 x 32 64.8 and 60.8        512   8 x 8 144 and 139, 1 x 64 87.7 and 84.8 (40 own rows: 76.7 and 73.7)
//   768 heads   12 x 8 233 and 218, 2 x 48 128 and 124 (40 own rows: 102 and 107)
//   1024 heads  16 x 8 322 and 309, 2 x 64 136 and 145 (40: 110 and 120), 64 x 2 over 4096 rows with 100 own 230 and 241
constexpr int kOwnHeads = 512;

template <int DT, int D>
struct ShShape {
  using T = Tile<DT, D>;
  static constexpr int kTiles = kStageBytes / (2 * T::kTileBytes);   // tiles of 32 rows in a stage
  static constexpr int kStageRows = 32 * kTiles;
  static constexpr int kHalves = 2 * kTiles;                          // half tiles, 16 rows each: within a page
  static constexpr int kMine = kHalves / kShWaves > 0 ? kHalves / kShWaves : 1;   // half tiles of a stage whose pages a wavefront holds
  static constexpr int kDBlocks = D / 32;
};

// The 16-byte slot of a row's chunk c is c ^ swizzle(row).  Keys: as the fragment reader has it.  bf16 values are read four rows by
// 64 bytes at a time, which lie in different banks only if neighbouring rows differ in the slot's upper bits (keys' order: 8 more
// cycles a read).
template <int DT, int D>
__device__ __forceinline__ int value_swizzle(int row) {
  if constexpr (DT == LAVA_F32) return row & 7;
  return D == 128 ? ((row & 3) << 2) | ((row >> 2) & 1) : ((row & 2) << 1) | ((row >> 2) & 1);
}

// 16 values of bf16 V^T as the left operand, for rows 16 s .. 16 s + 15 of a tile and columns 32 dblk ..: two reads of four rows
// each; at: this lane's address for rows 0 .. 3 of the tile and dblk 0 (a block is 64 bytes and so a bit of the slot, which the swizzle
// flips or not: an exclusive or); the second four lie 8 rows on.
template <int D, int S>
__device__ __forceinline__ void read_v(unsigned int at, u32x4 (&v)[D / 32]) {
  constexpr int R = D * 2, o = 16 * S * R;
  typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
  u32x2 x[D / 16];
  if constexpr (D == 128) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8 offset:%12\n\t"
        "ds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
        "ds_read_b64_tr_b16 %2, %9 offset:%12\n\t"
        "ds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
        "ds_read_b64_tr_b16 %4, %10 offset:%12\n\t"
        "ds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
        "ds_read_b64_tr_b16 %6, %11 offset:%12\n\t"
        "ds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
        : "v"(at), "v"(at ^ 64u), "v"(at ^ 128u), "v"(at ^ 192u), "n"(o), "n"(o + 8 * R)
        : "memory");
  } else {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %4 offset:%6\n\t"
        "ds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
        "ds_read_b64_tr_b16 %2, %5 offset:%6\n\t"
        "ds_read_b64_tr_b16 %3, %5 offset:%7\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
        : "v"(at), "v"(at ^ 64u), "n"(o), "n"(o + 8 * R)
        : "memory");
  }
#pragma unroll
  for (int d = 0; d < D / 32; ++d) v[d] = u32x4{x[2 * d].x, x[2 * d].y, x[2 * d + 1].x, x[2 * d + 1].y};
}

// Four 32-bit values at one offset from four addresses.
template <int OFF>
__device__ __forceinline__ void lds_read32x4_at(const unsigned int (&a)[4], unsigned int base, float (&o)[4]) {
  unsigned int x0 = a[0] + base, x1 = a[1] + base, x2 = a[2] + base, x3 = a[3] + base;
  asm volatile(
      "ds_read_b32 %0, %4 offset:%8\n\t"
      "ds_read_b32 %1, %5 offset:%8\n\t"
      "ds_read_b32 %2, %6 offset:%8\n\t"
      "ds_read_b32 %3, %7 offset:%8\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3])
      : "v"(x0), "v"(x1), "v"(x2), "v"(x3), "n"(OFF)
      : "memory");
}

// A tile's fragments from the address of this lane's first chunk: step j is 32 bytes on, before the swizzle.
template <int STEPS>
__device__ __forceinline__ void read_k(unsigned int at, u32x4 (&k)[STEPS]) {
#pragma unroll
  for (int j = 0; j < STEPS; j += 4)
    lds_read128x4(at ^ (32u * j), at ^ (32u * (j + 1)), at ^ (32u * (j + 2)), at ^ (32u * (j + 3)), k[j], k[j + 1], k[j + 2], k[j + 3]);
}

template <int DT, int D, bool OPT>
__global__ void __launch_bounds__(kShThreads, 2) shared_rows_kernel(const SharedArgs a) {
  using S = ShShape<DT, D>;
  using T = Tile<DT, D>;
  __shared__ __attribute__((aligned(1024))) u32x4 s_stage[2][kStageBytes / 16];   // (addresses are formed by exclusive or) keys' tiles, then values'; between units: float [kShWaves][32][D]
  __shared__ __attribute__((aligned(16))) int s_pos[2][OPT ? S::kStageRows : 4];
  __shared__ float s_m[kShWaves][32], s_l[kShWaves][32];
  __shared__ unsigned long long s_seen[kShWaves];
  __shared__ int s_wrong, s_next, s_first[kOwnHeads];        // the next unit; of every head the units of own rows before it
  const PagedDecodeArgs& p = a.p;
  const int lane = threadIdx.x & 63, wave = wave_index(), col = lane & 31, half = lane >> 5;
  const int n_items = a.n_items[0];
  auto stages_in = [](int rows) { return rows > 0 ? (int)(((unsigned int)rows + S::kStageRows - 1u) / S::kStageRows) : 0; };
  auto stages_of = [&](int i) { return i < n_items ? stages_in(a.items[i].rows) : 0; };
  const unsigned int wgs = gridDim.x;
  const bool windowed = OPT && p.window > 0;
  // Units of `share` stages of one item or head: no more units than workgroups where those are few; twice as many where parts of the
  // rows are out of the window, so that they are spread.
  auto share_of = [&](unsigned int total, unsigned int full) {
    const unsigned int cut = 2u * full <= wgs && !windowed ? wgs - full : 2u * wgs;
    return (int)((total + cut - 1u) / cut);
  };
  unsigned int total = 0u, full = 0u;
  for (int i = lane; i < n_items; i += 64) {
    const int n = stages_of(i);
    total += (unsigned int)n;
    full += n > 0 ? 1u : 0u;
  }
  total = lane_value(wave_incl(total), 63);
  full = lane_value(wave_incl(full), 63);
  const int share = total > 0u ? share_of(total, full) : 1;
  const int own_heads = a.own_here != 0 ? p.batch * p.H_kv : 0;   // <= kOwnHeads
  constexpr int kOwnEach = kOwnHeads / 64;
  unsigned int common_units = 0u, own_units = 0u;
  int own_share = 1;
  {
    unsigned int n = 0u;
    for (int i = lane; i < n_items; i += 64) n += (unsigned int)(stages_of(i) + share - 1) / (unsigned int)share;
    common_units = lane_value(wave_incl(n), 63);
  }
  if (own_heads > 0) {                                         // uniform; every wavefront finds the same
    int held[kOwnEach];
    unsigned int own = 0u, some = 0u;
#pragma unroll
    for (int c = 0; c < kOwnEach; ++c) held[c] = 64 * c + lane < own_heads ? a.rest_rows[64 * c + lane] : 0;
#pragma unroll
    for (int c = 0; c < kOwnEach; ++c) {
      held[c] = stages_in(held[c]);
      own += (unsigned int)held[c];
      some += held[c] > 0 ? 1u : 0u;
    }
    own = lane_value(wave_incl(own), 63);
    some = lane_value(wave_incl(some), 63);
    if (own > 0u) own_share = share_of(own, some);
#pragma unroll
    for (int c = 0; c < kOwnEach; ++c) {
      const unsigned int n = (unsigned int)(held[c] + own_share - 1) / (unsigned int)own_share, incl = wave_incl(n);
      if (wave == 0) s_first[64 * c + lane] = (int)(own_units + incl - n);
      own_units += lane_value(incl, 63);
    }
    __syncthreads();
  }
  const unsigned int all_units = common_units + own_units;

  TileDma<DT, D> dma;
  dma.init(lane);
  const unsigned int k_at = (unsigned int)(col * T::kRowBytes + ((half ^ (col & 7)) << 4));   // this lane's first chunk of a tile's row
  const unsigned int ring = lds_addr(&s_stage[0][0]);
  constexpr unsigned int kVOff = S::kTiles * T::kTileBytes;
  // bf16: where this lane's four columns of row 4 half + (lane % 16) / 4 lie.  32 bits: this lane's column of rows 4 half + 0 .. 3.
  unsigned int v_at[4] = {0u, 0u, 0u, 0u};
  unsigned int v_off[TileDma<DT, D>::kVariants];               // of the values' direct-to-LDS loads, as TileDma has them for keys
  if constexpr (DT == LAVA_BF16) {
    const int i = lane & 15, r = 4 * half + (i >> 2), c = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    v_at[0] = (unsigned int)(r * T::kRowBytes + ((c ^ value_swizzle<DT, D>(r)) << 4) + 8 * (i & 1));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * half + e;
      v_at[e] = (unsigned int)(r * T::kRowBytes + (((col >> 2) ^ value_swizzle<DT, D>(r)) << 4) + 4 * (col & 3));
    }
  }
#pragma unroll
  for (int i = 0; i < TileDma<DT, D>::kVariants; ++i) {
    const int q = i * 64 + lane, row = q / T::kCpr, slot = q % T::kCpr;
    v_off[i] = (unsigned int)((row - i * TileDma<DT, D>::kRowsPerLoad) * T::kRowBytes + ((slot ^ value_swizzle<DT, D>(row)) << 4));
  }
  const float inv_cap = p.cap > 0.0f ? 1.0f / p.cap : 0.0f;
  const unsigned int window = p.window > 0 ? (unsigned int)p.window : 0x80000000u;

  for (unsigned int u = blockIdx.x; u < all_units;) {
    unsigned int next_unit = 0u;                               // of thread 0; asked for now, needed when this unit is done
    if (threadIdx.x == 0) next_unit = wgs + __hip_atomic_fetch_add(reinterpret_cast<unsigned int*>(&a.n_items[1]), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // ---------------- the unit: its item, its part of the item, where its rows go
    int item = -1, part = 0, units = 0, row0 = 0, unit_share = share;
    SharedItem it;
    if (u < common_units) {
      unsigned int at = 0u, rows = 0u;
      for (int i0 = 0; i0 < n_items && item < 0; i0 += 64) {
        const int n = (int)((unsigned int)(stages_of(i0 + lane) + share - 1) / (unsigned int)share);
        const int mine = n > 0 ? n * a.items[i0 + lane].n_seq * p.G : 0;
        const unsigned int incl = wave_incl((unsigned int)n), r_incl = wave_incl((unsigned int)mine);
        const unsigned long long after = __ballot(at + incl > u);
        if (after != 0ull) {
          const int l = __builtin_ctzll(after);
          item = i0 + l;
          units = (int)lane_value((unsigned int)n, l);
          part = (int)(u - (at + lane_value(incl, l) - (unsigned int)units));
          row0 = (int)(rows + lane_value(r_incl, l) - lane_value((unsigned int)mine, l));
        } else {
          at += lane_value(incl, 63);
          rows += lane_value(r_incl, 63);
        }
      }
      it = a.items[item];
      if (part == 0 && threadIdx.x == 0) a.parts[item] = SharedParts{row0, units};
    } else {
      const int v = (int)(u - common_units);
      int h = -1;
#pragma unroll
      for (int c = 0; c < kOwnEach; ++c)
        h += __popcll(__ballot(64 * c + lane < own_heads && s_first[64 * c + lane] <= v));   // heads without units share the next one's number
      const int end = h + 1 < own_heads ? s_first[h + 1] : (int)own_units;
      part = v - s_first[h];
      units = end - s_first[h];
      row0 = a.own_base + s_first[h] * p.G;
      unit_share = own_share;
      it.first_seq = it.lead = h / p.H_kv;
      it.n_seq = 1;
      it.head = h - it.first_seq * p.H_kv;
      it.rows = a.rest_rows[h];
      it.skip = a.skip[h];
      if (part == 0 && threadIdx.x == 0) a.own_parts[h] = SharedParts{row0, units};
    }
    const int q_rows = it.n_seq * p.G;
    const int row_tiles = q_rows <= 32 ? 1 : q_rows <= 64 ? 2 : q_rows <= 128 ? 4 : 8;
    const int rt = wave & (row_tiles - 1), kp = wave / row_tiles, key_parts = kShWaves / row_tiles;
    const int s0 = part * unit_share, s_all = stages_in(it.rows), s1 = s0 + unit_share < s_all ? s0 + unit_share : s_all;
    const int* table = p.block_table + ((long long)it.lead * p.H_kv + it.head) * p.max_blocks + it.skip;

    // ---------------- the queries of this lane's column: a sequence that holds nothing in this head has none, whatever stands there
    const int qr = rt * 32 + col;
    const bool there = qr < q_rows;
    const int q_seq = it.first_seq + (there ? qr / p.G : 0), q_head = it.head * p.G + (there ? qr % p.G : 0);
    const bool real = there && p.head_rows[(long long)q_seq * p.H_kv + it.head] != 0;
    u32x4 qf[T::kSteps];
#pragma unroll
    for (int j = 0; j < T::kSteps; ++j) qf[j] = reinterpret_cast<const u32x4*>(p.q)[((long long)q_seq * p.H + q_head) * T::kCpr + 2 * j + half];
    const int q_pos = OPT && p.pos != nullptr ? p.q_pos[q_seq] : 0;
    const float slope = OPT && p.slopes != nullptr ? p.slopes[q_head] * kLog2e : 0.0f;

    float m_run = -INFINITY, l_run = 0.0f;
    f32x16 acc[S::kDBlocks];
#pragma unroll
    for (int d = 0; d < S::kDBlocks; ++d) acc[d] = f32x16{0};
    if (threadIdx.x == 0) s_wrong = 0;
    __syncthreads();                                           // LDS is free, s_wrong is set

    // pages of this wavefront's half tiles of stages sb .. sb + 63, a lane each
    int page[S::kMine];
    auto load_pages = [&](int sb) {
#pragma unroll
      for (int x = 0; x < S::kMine; ++x) {
        const int hh = (wave + kShWaves * x) % S::kHalves, r = (sb + lane) * S::kStageRows + 16 * hh;
        page[x] = sb + lane < s1 && r < it.rows ? table[r >> p.page_shift] : -2;
      }
#pragma unroll
      for (int x = 0; x < S::kMine; ++x) {
        if (page[x] == -2) page[x] = 0;                        // behind the last row: masked, any page will do
        else if (page[x] < 0 || page[x] >= p.n_pages) {
          page[x] = 0;
          s_wrong = 2;
        }
      }
    };
    int pos_next[S::kMine] = {};
    auto issue = [&](int s, int sb, int buffer) {              // stage s of pages loaded from sb on
      u32x4* dst = s_stage[buffer];
#pragma unroll
      for (int x = 0; x < 4 * S::kTiles / kShWaves; ++x) {
        const int k = wave + kShWaves * x, hh = k % S::kHalves;
        const bool is_v = k >= S::kHalves;
        const int r = s * S::kStageRows + 16 * hh;
        const long long place = ((long long)(int)lane_value((unsigned int)page[x % S::kMine], s - sb) << p.page_shift) +
                                (r < it.rows ? r & ((1 << p.page_shift) - 1) : 0);
        const char* src = (is_v ? p.v : p.k) + place * T::kRowBytes;
        u32x4* to = dst + (is_v ? S::kTiles * T::kTileChunks : 0) + hh * (T::kTileChunks / 2);
#pragma unroll
        for (int i = 0; i < T::kLoads / 2; ++i)
          __builtin_amdgcn_global_load_lds((const LAVA_GLOBAL_AS void*)(src + i * 1024 + (is_v ? v_off : dma.loff)[i % TileDma<DT, D>::kVariants]),
                                           (LAVA_LDS_AS void*)(to + i * 64), 16, 0, 0);
        if (OPT && p.pos != nullptr && !is_v) pos_next[x % S::kMine] = p.pos[place + (lane & 15)];
      }
    };
    // The stages of sb .. sb + 63 that hold rows in the window of any of the item's queries, as bits.
    unsigned int reach = 0u, last = 0u;                        // last: the latest position; rows further back than `reach` are seen by nobody
    if (windowed) {
      int lo = 0x7fffffff, hi = -0x7fffffff - 1;
      for (int i = lane; i < it.n_seq; i += 64) {
        const int y = p.q_pos[it.first_seq + i];
        const bool holds = p.head_rows[(long long)(it.first_seq + i) * p.H_kv + it.head] != 0;
        lo = holds ? min(lo, y) : lo;
        hi = holds ? max(hi, y) : hi;
      }
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        lo = min(lo, __shfl_xor(lo, m));
        hi = max(hi, __shfl_xor(hi, m));
      }
      last = (unsigned int)hi;
      const unsigned int spread = (unsigned int)hi - (unsigned int)lo;
      reach = spread < 0x80000000u - window ? window + spread : 0x80000000u;
    }
    auto seen_from = [&](int sb) -> unsigned long long {
      const int here = s1 - sb;
      const unsigned long long all = here >= 64 ? ~0ull : (1ull << here) - 1ull;
      if (!windowed) return all;
      bool any = false;
#pragma unroll
      for (int x = 0; x < S::kMine; ++x) {
        const int hh = (wave + kShWaves * x) % S::kHalves, r = (sb + lane) * S::kStageRows + 16 * hh;
        if (lane >= here || r >= it.rows) continue;
        const u32x4* at = reinterpret_cast<const u32x4*>(p.pos + ((long long)page[x] << p.page_shift) + (r & ((1 << p.page_shift) - 1)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32x4 y = at[i];
#pragma unroll
          for (int e = 0; e < 4; ++e) any |= last - y[e] < reach;
        }
      }
      const unsigned long long mine = __ballot(any);
      if (lane == 0) s_seen[wave] = mine;
      __syncthreads();
      unsigned long long seen = 0ull;
      for (int w = 0; w < kShWaves; ++w) seen |= s_seen[w];
      __syncthreads();
      return seen & all;
    };

    int sb = s0;
    load_pages(sb);
    unsigned long long todo = seen_from(sb);
    auto next_stage = [&]() -> int {                           // -1: none left
      while (todo == 0ull) {                                   // uniform over the workgroup
        sb += 64;
        if (sb >= s1) return -1;
        load_pages(sb);
        todo = seen_from(sb);
      }
      const int j = __builtin_ctzll(todo);
      todo &= todo - 1ull;
      return sb + j;
    };
    int s = next_stage(), buffer = 0;
    if (s >= 0) issue(s, sb, buffer);
    // not before: the loads that this waits for are on their way with those of pages and positions (ragged windows 66.0 -> 65.4 us)
#pragma unroll
    for (int j = 0; j < T::kSteps; ++j) qf[j] = real ? qf[j] : u32x4{0u, 0u, 0u, 0u};
    while (s >= 0) {
      wait_vmcnt<0>();
      if (OPT && p.pos != nullptr) {
#pragma unroll
        for (int x = 0; x < S::kMine; ++x) {
          const int k = wave + kShWaves * x;
          if (k < S::kHalves && lane < 16) lds_write32(lds_addr(&s_pos[buffer][16 * k + lane]), __int_as_float(pos_next[x]));
        }
      }
      if (it.rows - s * S::kStageRows < S::kStageRows) {                 // uniform: rows behind the last one weigh nothing, whatever was there
#pragma unroll
        for (int x = 0; x < 4 * S::kTiles / kShWaves; ++x) {
          const int k = wave + kShWaves * x, hh = k % S::kHalves, left = it.rows - s * S::kStageRows - 16 * hh;
          if (k < S::kHalves || left >= 16) continue;          // keys: their logits are masked
          const unsigned int row = lds_addr(&s_stage[buffer][S::kTiles * T::kTileChunks + hh * (T::kTileChunks / 2)]) + (unsigned int)(lane >> 2) * T::kRowBytes;
          const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          if ((lane >> 2) >= left)
#pragma unroll
            for (int c = 0; c < T::kRowBytes / 64; ++c) lds_write128(row + (unsigned int)(16 * (4 * c + (lane & 3))), zero);
        }
      }
      lds_reads_done();
      __syncthreads();                                         // the stage is there, the other one free
      const int next = next_stage();
      if (next >= 0) issue(next, sb, buffer ^ 1);
      asm volatile("" ::: "memory");
      const unsigned int stage = ring + (unsigned int)buffer * kStageBytes;
      for (int t = kp; t < S::kTiles; t += key_parts) {
        const int r0 = s * S::kStageRows + 32 * t;             // first row of the tile
        if (r0 >= it.rows) break;                              // uniform
        f32x16 z = {0};
        {
          u32x4 kf[T::kSteps];
          read_k(stage + (unsigned int)t * T::kTileBytes + k_at, kf);
#pragma unroll
          for (int j = 0; j < T::kSteps; ++j) z = mfma_chunk<DT>(kf[j], qf[j], z);
        }
        float x[16];                                           // of rows 8 (v / 4) + 4 half + v % 4
        if (OPT && p.cap > 0.0f) {                             // uniform
          float most = 0.0f;
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            x[v] = z[v] * p.scale;
            most = fmaxf(most, fabsf(x[v]));
          }
          if (__ballot(!(most < 0.25f * p.cap)) == 0ull) {     // all near zero, as logits mostly are: without the exponential
#pragma unroll
            for (int v = 0; v < 16; ++v) x[v] = capped_near(x[v], p.cap * kLog2e, inv_cap);
          } else {
#pragma unroll
            for (int v = 0; v < 16; ++v) x[v] = capped(x[v], p.cap, inv_cap) * kLog2e;
          }
        } else {
#pragma unroll
          for (int v = 0; v < 16; ++v) x[v] = z[v] * a.c2;
        }
        if (OPT && p.pos != nullptr) {                         // uniform
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4) {
            u32x4 at;
            lds_read128(lds_addr(&s_pos[buffer][32 * t + 8 * v4 + 4 * half]), at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const unsigned int back = (unsigned int)q_pos - at[e];   // a later row: 2^31 and more
              const float y = x[4 * v4 + e] - slope * (float)back;
              x[4 * v4 + e] = back < window ? y : -INFINITY;
            }
          }
        }
        if (it.rows - r0 < 32) {                               // uniform: some are behind the last row
#pragma unroll
          for (int v = 0; v < 16; ++v) x[v] = r0 + 8 * (v / 4) + 4 * half + v % 4 < it.rows ? x[v] : -INFINITY;
        }
        float top = x[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) top = fmaxf(top, x[v]);
        {
          const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
          top = fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
        }
        if (__ballot(top > m_run + kSlack) != 0ull) {          // uniform: a maximum moves
          const float m_new = fmaxf(m_run, top), keep = m_new == -INFINITY ? 1.0f : fast_exp2(m_run - m_new);
          m_run = m_new;
          l_run *= keep;
#pragma unroll
          for (int d = 0; d < S::kDBlocks; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[d][v] *= keep;
        }
        const float base = m_run == -INFINITY ? 0.0f : m_run;
        float e[16], sum = 0.0f;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          e[v] = fast_exp2(x[v] - base);
          sum += e[v];
        }
        l_run += sum;
        const unsigned int values = stage + kVOff + (unsigned int)t * T::kTileBytes;
        if constexpr (DT == LAVA_BF16) {
          static_for<2>([&](auto sc) {
            constexpr int h = decltype(sc)::value;
            u32x4 parts[3];
            {
              u32x4 lo, hi;
#pragma unroll
              for (int v = 0; v < 4; ++v) {
                lo[v] = __float_as_uint(e[8 * h + v]);
                hi[v] = __float_as_uint(e[8 * h + 4 + v]);
              }
              split8(lo, hi, parts[0], parts[1], parts[2]);
            }
            u32x4 vt[S::kDBlocks];
            read_v<D, h>(values + v_at[0], vt);
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll
              for (int d = 0; d < S::kDBlocks; ++d) acc[d] = mfma_bf16(vt[d], parts[k], acc[d]);
          });
        } else {
          static_for<4 * S::kDBlocks>([&](auto ic) {
            constexpr int v4 = decltype(ic)::value / S::kDBlocks, d = decltype(ic)::value % S::kDBlocks;
            float vv[4];
            lds_read32x4_at<8 * v4 * T::kRowBytes + 128 * d>(v_at, values, vv);
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vv[k], e[4 * v4 + k], acc[d], 0, 0, 0);
          });
        }
      }
      lds_reads_done();
      s = next;
      buffer ^= 1;
    }
    // ---------------- the unit's part: wavefronts with the same queries put together
    l_run = add_halves(l_run);
    bool wrong = !(l_run < INFINITY);
#pragma unroll
    for (int d = 0; d < S::kDBlocks; ++d)
#pragma unroll
      for (int v = 0; v < 16; ++v) wrong |= !(fabsf(acc[d][v]) < INFINITY);
    if (wrong && real) atomicOr(&a.head_marked[(long long)q_seq * p.H_kv + it.head], 1);
    __syncthreads();                                           // every wavefront is done with the stages
    constexpr int kChunks = D / 4;                             // 16-byte chunks of an output row
    float* s_acc = reinterpret_cast<float*>(&s_stage[0][0]);
    if (half == 0) {
      s_m[wave][col] = m_run;
      s_l[wave][col] = l_run;
    }
#pragma unroll
    for (int d = 0; d < S::kDBlocks; ++d)
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        const int c = 8 * d + 2 * v4 + half;                   // columns 32 d + 8 v4 + 4 half ..
        *reinterpret_cast<float4*>(s_acc + (wave * 32 + col) * D + 4 * (c ^ (col & (kChunks - 1)))) =
            make_float4(acc[d][4 * v4], acc[d][4 * v4 + 1], acc[d][4 * v4 + 2], acc[d][4 * v4 + 3]);
      }
    __syncthreads();
    if (threadIdx.x == 0) {
      if (s_wrong != 0) atomicOr(item >= 0 ? &a.marked[item] : &a.head_marked[it.first_seq * p.H_kv + it.head], s_wrong);
      s_next = (int)next_unit;
    }
    const long long out0 = (long long)row0 + (long long)part * q_rows;
    for (int i = threadIdx.x; i < q_rows * kChunks; i += kShThreads) {
      const int r = i / kChunks, c = i - r * kChunks, w0 = r >> 5, cr = r & 31;
      float M = -INFINITY;
      for (int k = 0; k < key_parts; ++k) M = fmaxf(M, s_m[w0 + k * row_tiles][cr]);
      const float base = M == -INFINITY ? 0.0f : M;
      float L = 0.0f;
      float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      for (int k = 0; k < key_parts; ++k) {
        const int w = w0 + k * row_tiles;
        const float wgt = fast_exp2(s_m[w][cr] - base);
        const float4 y = *reinterpret_cast<const float4*>(s_acc + (w * 32 + cr) * D + 4 * (c ^ (cr & (kChunks - 1))));
        L += wgt * s_l[w][cr];
        sum.x += wgt * y.x;
        sum.y += wgt * y.y;
        sum.z += wgt * y.z;
        sum.w += wgt * y.w;
      }
      *reinterpret_cast<float4*>(a.part_acc + (out0 + r) * D + 4 * c) = sum;
      if (c == 0) a.part_ml[out0 + r] = make_float2(M, L);
    }
    __syncthreads();                                           // the next unit may use LDS
    u = (unsigned int)__builtin_amdgcn_readfirstlane(s_next);
  }
}

// ---------------------------------------------------------------- merge
constexpr int kMergeThreads = 256;

// One head's output from all its rows, eight that are seen at a time: where a value in a masked row may be infinite or no number.  Rare, and
// slow beside the products: 131072 rows of 4 queries with an infinity among the values 26 ms (one row at a time 95).  A sum that is no number ends
// it, so that a query that is none costs 40 us beside 64 sequences of that length (to the last row: 128 ms).
template <int DT, int D>
__device__ __forceinline__ void whole_head(const SharedArgs& a, int b, int g, float* s_red) {
  const PagedDecodeArgs& p = a.p;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rows = p.head_rows[(long long)b * p.H_kv + g];
  constexpr int kWaves = kMergeThreads / 64, kEach = D / 64, kAtOnce = 8;
  const int* table = p.block_table + ((long long)b * p.H_kv + g) * p.max_blocks;
  const int q_pos = p.pos != nullptr ? p.q_pos[b] : 0;
  const unsigned int window = p.window > 0 ? (unsigned int)p.window : 0x80000000u;
  auto load = [&](const char* from, long long place, float (&y)[kEach]) {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const long long at = place * D + lane * kEach + e;
      y[e] = DT == LAVA_BF16 ? __uint_as_float((unsigned int)reinterpret_cast<const unsigned short*>(from)[at] << 16)
                             : reinterpret_cast<const float*>(from)[at];
    }
  };
  for (int t = 0; t < p.G; ++t) {
    const long long row = (long long)b * p.H + (long long)g * p.G + t;
    const float slope = p.slopes != nullptr ? p.slopes[g * p.G + t] * kLog2e : 0.0f;
    float q[kEach], acc[kEach] = {}, M = -INFINITY, L = 0.0f;
    load(p.q, row, q);
    bool bad = false;
    for (unsigned int r0 = 64u * wave; r0 < (unsigned int)rows; r0 += 64u * kWaves) {   // (a head may have 2^31 rows, nearly)
      // a lane a row: where it lies and whether it is seen
      const unsigned int r = r0 + lane;
      const bool held = r < (unsigned int)rows;
      const int page = held ? table[r >> p.page_shift] : 0;
      const bool there = held && page >= 0 && page < p.n_pages;
      const long long place = there ? ((long long)page << p.page_shift) + (int)(r & ((1u << p.page_shift) - 1u)) : 0;
      const unsigned int back = p.pos != nullptr && there ? (unsigned int)q_pos - (unsigned int)p.pos[place] : 0u;
      bad |= __ballot(held && !there) != 0ull;
      unsigned long long todo = __ballot(there && back < window);
      while (todo != 0ull) {                                   // uniform; kAtOnce of the rows that are seen
        bool on[kAtOnce];
        unsigned int off[kAtOnce];
        float k[kAtOnce][kEach], v[kAtOnce][kEach], x[kAtOnce], top = M;
        int j = 0;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          on[i] = todo != 0ull;
          j = on[i] ? __builtin_ctzll(todo) : j;
          todo &= todo - 1ull;
          const long long at = lane_value64(place, j);
          off[i] = lane_value(back, j);
          load(p.k, at, k[i]);
          load(p.v, at, v[i]);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          x[i] = 0.0f;
#pragma unroll
          for (int e = 0; e < kEach; ++e) x[i] = fmaf(q[e], k[i][e], x[i]);
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1)
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) x[i] += __shfl_xor(x[i], m);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          x[i] = p.cap > 0.0f ? capped(x[i] * p.scale, p.cap, 1.0f / p.cap) * kLog2e : x[i] * a.c2;
          x[i] = on[i] ? x[i] - slope * (float)off[i] : -INFINITY;
          top = fmaxf(top, x[i]);
        }
        const float base = top == -INFINITY ? 0.0f : top, keep = fast_exp2(M - base);
        M = top;
        L *= keep;
#pragma unroll
        for (int e = 0; e < kEach; ++e) acc[e] *= keep;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          if (!on[i]) continue;                                // uniform
          const float w = fast_exp2(x[i] - base);
          L += w;
#pragma unroll
          for (int e = 0; e < kEach; ++e) acc[e] += w * v[i][e];
        }
      }
      if (isnan(L)) break;                                     // uniform: so is the head's sum, whatever follows
    }
    if (bad) L = NAN;
    __syncthreads();
    if (lane == 0) {
      s_red[2 * wave] = M;
      s_red[2 * wave + 1] = L;
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) s_red[2 * kWaves + wave * D + lane * kEach + e] = acc[e];
    __syncthreads();
    if ((int)threadIdx.x < D) {
      float top = -INFINITY, sum = 0.0f, y = 0.0f;
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_red[2 * w]);
      const float base = top == -INFINITY ? 0.0f : top;
      for (int w = 0; w < kWaves; ++w) {
        const float wgt = fast_exp2(s_red[2 * w] - base);
        sum += wgt * s_red[2 * w + 1];
        y += wgt * s_red[2 * kWaves + w * D + threadIdx.x];
      }
      p.out[row * D + threadIdx.x] = sum == 0.0f ? 0.0f : y / sum;
      if (threadIdx.x == 0 && p.lse != nullptr) p.lse[row] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
    }
  }
}

template <int DT, int D>
__global__ void __launch_bounds__(kMergeThreads) shared_merge_kernel(const SharedArgs a) {
  __shared__ float s_red[(kMergeThreads / 64) * (D + 2)], s_base[8], s_own[8], s_sum[8];
  const PagedDecodeArgs& p = a.p;
  const int b = blockIdx.x / p.H_kv, g = blockIdx.x - b * p.H_kv;
  const int item = a.item_of[blockIdx.x];
  const bool here = a.own_here != 0;
  const long long row0 = (long long)b * p.H + (long long)g * p.G;
  if (item < 0 && !here) return;                               // nothing in common: the own rows were all
  const int rest = here ? a.rest_rows[blockIdx.x] : 0;
  const int marked = (item >= 0 ? a.marked[item] : 0) | a.head_marked[blockIdx.x];
  if (marked == 1) {                                           // no page was wrong: only values
    whole_head<DT, D>(a, b, g, s_red);
    return;
  }
  // parts 0 .. n_common - 1 are the common rows', n_common .. n - 1 the own ones'
  int n_common = 0, n = 0, common_step = 0;
  long long common0 = 0, own0 = 0;
  if (item >= 0) {
    const SharedItem it = a.items[item];
    const SharedParts x = a.parts[item];
    common_step = it.n_seq * p.G;
    common0 = x.row + (long long)(b - it.first_seq) * p.G;
    n = n_common = x.units;
  }
  if (rest > 0) {
    const SharedParts x = a.own_parts[blockIdx.x];
    own0 = x.row;
    n += x.units;
  }
  auto row_of = [&](int u, int t) {
    return u < n_common ? common0 + t + (long long)u * common_step : own0 + t + (long long)(u - n_common) * p.G;
  };
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // a wavefront a query: the maximum over its parts, then their weights
  for (int t = wave; t < p.G; t += kMergeThreads / 64) {
    const float2 own = here ? make_float2(-INFINITY, 0.0f) : a.rest_sums[row0 + t];
    float M = own.x, L = 0.0f;
    for (int u = lane; u < n; u += 64) M = fmaxf(M, a.part_ml[row_of(u, t)].x);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) M = fmaxf(M, __shfl_xor(M, m));
    const float base = M == -INFINITY ? 0.0f : M;
    for (int u = lane; u < n; u += 64) {
      const float2 ml = a.part_ml[row_of(u, t)];
      L += fast_exp2(ml.x - base) * ml.y;
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) L += __shfl_xor(L, m);
    const float wgt = fast_exp2(own.x - base) * own.y;         // NaN: a page that is not in the pool, or rows that cannot be
    L += wgt;
    if (marked != 0 || rest < 0) L = NAN;                      // the same
    if (lane == 0) {
      s_base[t] = base;
      s_own[t] = wgt;
      s_sum[t] = L;
      if (p.lse != nullptr) p.lse[row0 + t] = L == 0.0f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
    }
  }
  __syncthreads();
  constexpr int kLoads = 8;
  for (int i = threadIdx.x; i < p.G * (D / 4); i += kMergeThreads) {
    const int t = i / (D / 4), c = i - t * (D / 4);
    const float base = s_base[t], L = s_sum[t], wgt = s_own[t];
    float4* out = reinterpret_cast<float4*>(p.out + (row0 + t) * D) + c;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (!here) {
      const float4 mine = *out;
      sum = make_float4(wgt * mine.x, wgt * mine.y, wgt * mine.z, wgt * mine.w);
    }
    for (int u0 = 0; u0 < n; u0 += kLoads) {
      float m[kLoads];
      float4 y[kLoads];
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {                       // behind the last part: the last one, at no weight
        const long long r = row_of(u0 + u < n ? u0 + u : n - 1, t);
        m[u] = a.part_ml[r].x;
        y[u] = *reinterpret_cast<const float4*>(a.part_acc + r * D + 4 * c);
      }
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const float w = u0 + u < n ? fast_exp2(m[u] - base) : 0.0f;
        sum.x += w * y[u].x;
        sum.y += w * y[u].y;
        sum.z += w * y[u].z;
        sum.w += w * y[u].w;
      }
    }
    *out = L == 0.0f ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : make_float4(sum.x / L, sum.y / L, sum.z / L, sum.w / L);
  }
}

bool own_is_here(const lava_layer_desc& d, int32_t batch) { return (int64_t)batch * d.n_kv_heads <= kOwnHeads; }

struct SharedLayout {
  size_t off_items, off_parts, off_own_parts, off_marked, off_head_marked, off_item_of, off_rest_rows, off_skip, off_rest_table, off_rest_sums, off_ml, off_acc;
  size_t off_decode, bytes, own_base;
};
SharedLayout shared_layout(const lava_layer_desc& d, int32_t batch, int32_t max_blocks) {
  const size_t heads = (size_t)batch * d.n_kv_heads, G = d.n_q_heads / d.n_kv_heads;
  const size_t widest = batch * G < (size_t)kShRows ? batch * G : (size_t)kShRows;
  // parts: `cut` units of whole shares at most, of the widest items, and one more unit an item; the same of the heads' own rows
  const size_t most = 2 * (size_t)device_cus(), all = (size_t)batch * d.n_q_heads;
  SharedLayout l;
  l.own_base = most * widest + all;
  const size_t rows = l.own_base + (own_is_here(d, batch) ? most * G + all : 0);
  l.off_items = align_up(2 * sizeof(int));
  l.off_parts = l.off_items + align_up(heads * sizeof(SharedItem));
  l.off_own_parts = l.off_parts + align_up(heads * sizeof(SharedParts));
  l.off_marked = l.off_own_parts + align_up(heads * sizeof(SharedParts));
  l.off_head_marked = l.off_marked + align_up(heads * 4);
  l.off_item_of = l.off_head_marked + align_up(heads * 4);
  l.off_rest_rows = l.off_item_of + align_up(heads * 4);
  l.off_skip = l.off_rest_rows + align_up(heads * 4);
  l.off_rest_table = l.off_skip + align_up(heads * 4);
  l.off_rest_sums = l.off_rest_table + (own_is_here(d, batch) ? 0 : align_up(heads * max_blocks * 4));
  l.off_ml = l.off_rest_sums + (own_is_here(d, batch) ? 0 : align_up((size_t)batch * d.n_q_heads * sizeof(float2)));
  l.off_acc = l.off_ml + align_up(rows * sizeof(float2));
  l.off_decode = l.off_acc + align_up(rows * d.head_dim * sizeof(float));
  l.bytes = l.off_decode + paged_decode_bytes(d);
  return l;
}

// A stage and the next one take more than half of a compute unit's LDS: one workgroup each.
template <int DT, int D>
int32_t launch_rows(const SharedArgs& a, hipStream_t s) {
  ProfScope ps(KID_SHARED_DECODE, s);
  const dim3 wgs((unsigned)device_cus());
  if (a.p.pos != nullptr || a.p.cap > 0.0f)
    hipLaunchKernelGGL((shared_rows_kernel<DT, D, true>), wgs, dim3(kShThreads), 0, s, a);
  else
    hipLaunchKernelGGL((shared_rows_kernel<DT, D, false>), wgs, dim3(kShThreads), 0, s, a);
  return launch_status();
}

template <int DT, int D>
int32_t launch_merge(const SharedArgs& a, hipStream_t s) {
  ProfScope ps(KID_SHARED_MERGE, s);
  hipLaunchKernelGGL((shared_merge_kernel<DT, D>), dim3((unsigned)(a.p.batch * a.p.H_kv)), dim3(kMergeThreads), 0, s, a);
  return launch_status();
}

// Tables that have room for no more bytes of keys and values than this, counted once for every sequence, are decoded sequence by sequence: the
// step over pages reads them, from the last-level cache mostly, before three launches have found out what is common.  bf16, d_h 128,
// 8 KV heads, apart and shared: 8 sequences of 4096 rows (138 MB) 24 and 36 us, 16 (277 MB) 35 and 40, 8 of 16384 (541 MB) 56 and 40,
// 4 groups of 8 of 4096 (554 MB) 55 and 41; 32 bits: 8 of 4096 (277 MB) 48 and 50, 4 of 16384 (541 MB) 80 and 76.  Room is all that the host
// knows: tables with room for much more than they hold (4 sequences of 1024 rows a head, room for 131072) take 24 us where narrow ones take 13.
constexpr long long kApartBytes = 400000000;

}  // namespace

size_t shared_decode_bytes(const lava_layer_desc& d, int32_t batch, int32_t max_blocks) { return shared_layout(d, batch, max_blocks).bytes; }

int32_t launch_shared_decode(const lava_layer_desc& d, const PagedDecodeArgs& p, int32_t n_groups, const int32_t* group_start, void* ws,
                             hipStream_t s) {
  const SharedLayout l = shared_layout(d, p.batch, p.max_blocks);
  char* w = static_cast<char*>(ws);
  const long long row_bytes = 2LL * d.head_dim * (d.dtype == LAVA_BF16 ? 2 : 4);
  const double room = (double)p.batch * p.H_kv * ((double)p.max_blocks * (1 << p.page_shift)) * row_bytes;
  if (n_groups == p.batch || room <= (double)kApartBytes) return launch_paged_decode(d, p, w + l.off_decode, s);
  SharedArgs a;
  a.p = p;
  a.n_groups = n_groups;
  a.group_start = group_start;
  a.c2 = p.scale * kLog2e;
  a.n_items = reinterpret_cast<int*>(w);
  a.items = reinterpret_cast<SharedItem*>(w + l.off_items);
  a.parts = reinterpret_cast<SharedParts*>(w + l.off_parts);
  a.own_here = own_is_here(d, p.batch) ? 1 : 0;
  a.own_base = (int)l.own_base;
  a.own_parts = reinterpret_cast<SharedParts*>(w + l.off_own_parts);
  a.marked = reinterpret_cast<int*>(w + l.off_marked);
  a.head_marked = reinterpret_cast<int*>(w + l.off_head_marked);
  a.skip = reinterpret_cast<int*>(w + l.off_skip);
  a.item_of = reinterpret_cast<int*>(w + l.off_item_of);
  a.rest_rows = reinterpret_cast<int*>(w + l.off_rest_rows);
  a.rest_table = reinterpret_cast<int*>(w + l.off_rest_table);
  a.rest_sums = reinterpret_cast<float2*>(w + l.off_rest_sums);
  a.part_ml = reinterpret_cast<float2*>(w + l.off_ml);
  a.part_acc = reinterpret_cast<float*>(w + l.off_acc);
  {
    ProfScope ps(KID_SHARED_PLAN, s);
    hipLaunchKernelGGL(shared_plan_kernel, dim3((unsigned)(n_groups * p.H_kv)), dim3(kPlanShThreads), 0, s, a);
  }
  int32_t st = launch_status();
  const bool bf16 = d.dtype == LAVA_BF16, wide = d.head_dim == 128;
  if (st == LAVA_OK)
    st = bf16 ? (wide ? launch_rows<LAVA_BF16, 128>(a, s) : launch_rows<LAVA_BF16, 64>(a, s))
              : (wide ? launch_rows<LAVA_F32, 128>(a, s) : launch_rows<LAVA_F32, 64>(a, s));
  if (st == LAVA_OK && a.own_here == 0) {
    PagedDecodeArgs own = p;
    own.block_table = a.rest_table;
    own.head_rows = a.rest_rows;
    own.sums = a.rest_sums;
    st = launch_paged_decode(d, own, w + l.off_decode, s);
  }
  if (st == LAVA_OK)
    st = bf16 ? (wide ? launch_merge<LAVA_BF16, 128>(a, s) : launch_merge<LAVA_BF16, 64>(a, s))
              : (wide ? launch_merge<LAVA_F32, 128>(a, s) : launch_merge<LAVA_F32, 64>(a, s));
  return st;
}

}  // namespace lava
