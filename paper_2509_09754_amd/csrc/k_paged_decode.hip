// Decode-step attention over the pages of the paged cache: out[h] = Softmax(z[h]) V_g over the rows that head g holds, z =
// scale <q, k>, optionally capped (cap tanh(z / cap)), biased by distance and restricted to a window of positions.
//
// The work is one line of 32-row tiles, head after head through the whole batch.  It is cut into equal shares, one per workgroup
// and as many workgroups as the device holds at a time, whatever the lengths: a ragged batch, a long sequence alone and a
// padded one all end together, and the host needs to know no length.  A share is a run of tiles that may end in one head
// and go on in the next; every workgroup finds its own with one pass over the row counts (an exclusive sum of 256 threads).
//
// Inside a share's part of one head the wavefronts take tiles in turn.  K goes through a wavefront's own LDS ring with
// direct-to-LDS loads, two tiles ahead, V straight into registers, one tile ahead (a lane owns the same columns of every row):
//   logits   K_tile x Q^T on the matrix cores (the G heads are G columns of the 32-wide operand; exact products, fp32 sums)
//   softmax  online, in the exp2 domain, per head, kept in the column's lanes
//   output   acc[head][columns of this lane] += p[row][head] * V[row][columns], p broadcast through LDS in fp32; V is never
//            rounded
// Pages: the numbers of a wavefront's next 64 tiles are held by its lanes, one each (two for pages of half a tile), and become
// scalars when their tile is requested, so that the table costs one trip to memory per 64 tiles.  With positions the same
// lanes find out which rows of their tiles are seen: tiles without any are not requested.
//
// A head inside one share is finished there; otherwise each workgroup publishes its part (maximum, sum, output) and the one
// that finds all parts of the head published merges them in order.  Flags and tags are those of the decode step over the packed cache
// (xblock.h): a flag counts only if it equals the call's tag, whoever merges a head clears its flags, nobody waits.
//
// Bound by HBM: 2 * d_h * elem bytes a row.
#include <math.h>

#include "common.h"
#include "decode_parts.h"
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
__device__ __forceinline__ long long part_slot(long long w0, int u) { return u == 0 ? 2 * w0 + 1 : 2 * (w0 + u); }

// Tiles of head hb; -1: its row count is none.
__device__ __forceinline__ int head_tiles(const PagedDecodeArgs& a, int rows) {
  if (rows < 0 || rows > (long long)a.max_blocks << a.page_shift) return -1;
  return (int)(((long long)rows + kTileKeys - 1) / kTileKeys);
}

// Exclusive sum over the workgroup's threads and the sum over all.
__device__ __forceinline__ long long share_scan(long long x, long long* s_part, long long* total) {
  const int lane = threadIdx.x & 63, wave = wave_index();
  long long incl = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned int lo = __shfl_up((unsigned int)incl, d), hi = __shfl_up((unsigned int)(incl >> 32), d);
    if (lane >= d) incl += (long long)(((unsigned long long)hi << 32) | lo);
  }
  if (lane == 63) s_part[wave] = incl;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kDecWaves; ++w) {
    const long long p = s_part[w];
    if (w < wave) before += p;
    all += p;
  }
  *total = all;
  return before + incl - x;
}

// cap * tanh(z / cap): near zero by its series (the quotient of exponentials would cancel), else from e^(-2 |z / cap|).
__device__ __forceinline__ float capped(float z, float cap, float inv_cap) {
  const float y = z * inv_cap, a = fabsf(y), s = y * y;
  float series = fmaf(s, 2.1869489e-2f, -5.3968254e-2f);             // 62 / 2835, -17 / 315
  series = fmaf(s, series, 1.3333333e-1f);
  series = fmaf(s, series, -3.3333333e-1f);
  series = fmaf(a * s, series, a);
  const float t = fast_exp2(a * (-2.0f * kLog2e));
  const float far = (1.0f - t) * __builtin_amdgcn_rcpf(1.0f + t);
  return cap * copysignf(a < 0.25f ? series : far, y);
}

// A value that is the same in every lane, as a scalar.
__device__ __forceinline__ long long uniform64(long long x) { return lane_value64(x, 0); }

// a / b for 0 <= a < 2^52, b > 0 (a quotient of doubles is off by less than one).
__device__ __forceinline__ long long quotient(long long a, long long b) {
  long long q = (long long)((double)a / (double)b);
  if (q * b > a) --q;
  if ((q + 1) * b <= a) ++q;
  return q;
}

// The parts of one head, in order.
constexpr int kPartChunk = 32;
template <int D, int GP>
__device__ __forceinline__ void merge_parts(const PagedArgs& a, int b, int g, long long w0, int parts, float2 (*s_ml)[GP]) {
  constexpr int kPairs = GP * D / 2, kOut = (kPairs + kDecThreads - 1) / kDecThreads;
  float M[kOut], L[kOut];
  float2 sum[kOut];
#pragma unroll
  for (int j = 0; j < kOut; ++j) { M[j] = -INFINITY; L[j] = 0.0f; sum[j] = make_float2(0.0f, 0.0f); }
  for (int c0 = 0; c0 < parts; c0 += kPartChunk) {
    const int nu = parts - c0 < kPartChunk ? parts - c0 : kPartChunk;
    float2 pv[kOut][16];
    auto load_parts = [&](int u0) {
#pragma unroll
      for (int j = 0; j < kOut; ++j) {
        const int idx = 2 * ((int)threadIdx.x + kDecThreads * j);
#pragma unroll
        for (int u = 0; u < 16; ++u)
          pv[j][u] = idx < GP * D && u0 + u < nu
                         ? ld_dev_f2(reinterpret_cast<const float2*>(a.part_acc + part_slot(w0, c0 + u0 + u) * GP * D + idx))
                         : make_float2(0.0f, 0.0f);
      }
    };
    load_parts(0);
    for (int i = threadIdx.x; i < nu * GP; i += kDecThreads) s_ml[i / GP][i % GP] = ld_dev_f2(&a.part_ml[part_slot(w0, c0 + i / GP) * GP + i % GP]);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kOut; ++j) {
      const int t = 2 * ((int)threadIdx.x + kDecThreads * j) / D;
      if (t >= GP) continue;
      float mc = s_ml[0][t].x;
      for (int u = 1; u < nu; ++u) mc = fmaxf(mc, s_ml[u][t].x);
      const float m_new = fmaxf(M[j], mc), base = m_new == -INFINITY ? 0.0f : m_new;   // -inf: nothing seen so far
      const float keep = fast_exp2(M[j] - base);
      M[j] = m_new;
      L[j] *= keep;
      sum[j].x *= keep;
      sum[j].y *= keep;
    }
    for (int u0 = 0; u0 < nu; u0 += 16) {
      if (u0 > 0) load_parts(u0);
#pragma unroll
      for (int j = 0; j < kOut; ++j) {
        const int t = 2 * ((int)threadIdx.x + kDecThreads * j) / D;
        if (t >= GP) continue;
        const float base = M[j] == -INFINITY ? 0.0f : M[j];
#pragma unroll
        for (int u = 0; u < 16; ++u) {
          if (u0 + u < nu) {
            const float2 st = s_ml[u0 + u][t];
            const float wgt = fast_exp2(st.x - base);
            L[j] += wgt * st.y;
            sum[j].x += wgt * pv[j][u].x;
            sum[j].y += wgt * pv[j][u].y;
          }
        }
      }
    }
    __syncthreads();                                         // the next chunk overwrites s_ml
  }
#pragma unroll
  for (int j = 0; j < kOut; ++j) {
    const int idx = 2 * ((int)threadIdx.x + kDecThreads * j), t = idx / D, e = idx % D;
    if (t >= a.p.G) continue;
    const long long row = (long long)b * a.p.H + (long long)g * a.p.G + t;
    const bool none = L[j] == 0.0f;                          // every row masked
    a.p.out[row * D + e] = none ? 0.0f : sum[j].x / L[j];
    a.p.out[row * D + e + 1] = none ? 0.0f : sum[j].y / L[j];
    if (a.p.lse != nullptr && e == 0) a.p.lse[row] = none ? -INFINITY : (M[j] + log2f(L[j])) * 0.6931471805599453f;
  }
}

template <int DT, int D, int GP, bool POS>
__global__ void __launch_bounds__(kDecThreads) paged_decode_kernel(PagedArgs a) {
  using S = DecShape<DT, D>;
  using T = Tile<DT, D>;
  constexpr int kStages = S::kStages;
  constexpr int kDpl = S::kDpl;
  __shared__ u32x4 s_tile[kDecWaves][kStages][T::kTileChunks];   // between heads: float [kDecWaves][GP][D]
  constexpr int kPs = GP < 4 ? 4 : GP;                      // floats per row in s_p (one or two 128-bit reads)
  __shared__ __attribute__((aligned(16))) float s_p[kDecWaves][kTileKeys + 1][kPs];   // probabilities; row 32: rescale factors
  __shared__ float s_m[kDecWaves][GP], s_l[kDecWaves][GP];
  __shared__ long long s_part[kDecWaves], s_start;
  __shared__ int s_head, s_flag, s_bad;

  const PagedDecodeArgs& p = a.p;
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int n_heads = p.batch * p.H_kv;
  const int shift = p.page_shift, page_mask = (1 << shift) - 1;

  // ---------------- this workgroup's share
  const int per = (n_heads + kDecThreads - 1) / kDecThreads;   // heads a thread adds up
  long long mine = 0;
  const int h_first = (int)threadIdx.x * per;
  for (int i = 0; i < per; ++i) {
    const int t = h_first + i < n_heads ? head_tiles(p, p.head_rows[h_first + i]) : 0;
    mine += t > 0 ? t : 0;
  }
  if (threadIdx.x == 0) s_bad = 0;
  long long total;
  const long long before = share_scan(mine, s_part, &total);
  total = uniform64(total);
  // heads that hold nothing, or whose count is none, belong to nobody's share
  for (int h0 = 0; h0 < n_heads; h0 += gridDim.x * 64) {
    const int hb = h0 + (int)blockIdx.x + (int)gridDim.x * lane;
    const int t = hb < n_heads ? head_tiles(p, p.head_rows[hb]) : 1;
    unsigned long long todo = __ballot(t <= 0);
    while (todo != 0ull) {
      const int l = __builtin_ctzll(todo);
      todo &= todo - 1ull;
      const float x = (int)lane_value((unsigned int)t, l) < 0 ? NAN : 0.0f;
      const int hx = h0 + (int)blockIdx.x + (int)gridDim.x * l, b = hx / p.H_kv;
      const long long row0 = (long long)b * p.H + (long long)(hx - b * p.H_kv) * p.G;
      for (int i = threadIdx.x; i < p.G * D; i += kDecThreads) p.out[row0 * D + i] = x;
      if (p.lse != nullptr && (int)threadIdx.x < p.G) p.lse[row0 + threadIdx.x] = x == 0.0f ? -INFINITY : x;
    }
  }
  // a share is at least four tiles, one per wavefront, unless the heads are shorter than that
  long long share = uniform64(quotient(total + gridDim.x - 1, gridDim.x));
  if (share < 4) {
    const long long least = total >= 4ll * n_heads ? 4 : total >= 3ll * n_heads ? 3 : total >= 2ll * n_heads ? 2 : 1;
    if (share < least) share = least;
  } else {
    share = (share + 3) & ~3ll;
  }
  const long long t0 = (long long)blockIdx.x * share;
  const long long t1 = t0 + share < total ? t0 + share : total;
  if (t0 >= total) return;
  if (mine > 0 && before <= t0 && t0 < before + mine) {      // one thread's heads hold the first tile
    long long at = before;
    for (int i = 0; i < per; ++i) {
      const int t = h_first + i < n_heads ? head_tiles(p, p.head_rows[h_first + i]) : 0;
      if (t <= 0) continue;
      if (t0 < at + t) {
        s_head = h_first + i;
        s_start = at;
        break;
      }
      at += t;
    }
  }
  __syncthreads();
  int hb = (int)lane_value((unsigned int)s_head, 0);
  long long head_start = uniform64(s_start);                 // tiles before this head

  using VRaw = typename RawBits<S::kBpl>::type;
  TileDma<DT, D> dma;
  dma.init(lane);
  u32x4* ring = s_tile[wave][0];
  FragReader<DT, D> frags;
  frags.init_at(lane, lds_addr(ring));
  const unsigned int p_addr = lds_addr(&s_p[wave][0][0]);
  const int col = lane & 31, half = lane >> 5;
  const unsigned int p_col = p_addr + (unsigned int)(col * 4);                  // row 0 of s_p, this head's column
  const unsigned int p_mine = p_col + (unsigned int)(4 * half * kPs * 4);       // first row this lane's results cover
  const unsigned int v_lane = (unsigned int)lane * S::kBpl;   // a row is a uniform address plus this
  const float inv_cap = p.cap > 0.0f ? 1.0f / p.cap : 0.0f;
  const unsigned int window = p.window > 0 ? (unsigned int)p.window : 0x80000000u;

  for (long long t = t0; t < t1;) {
    const int rows = p.head_rows[hb];
    const int tiles = head_tiles(p, rows);
    if (tiles <= 0) { ++hb; continue; }                       // uniform
    const int b = hb / p.H_kv, g = hb - b * p.H_kv;
    const int ta = (int)(t - head_start), tb = head_start + tiles < t1 ? tiles : (int)(t1 - head_start);   // tiles of the head
    const int* __restrict__ table = p.block_table + (long long)hb * p.max_blocks;
    const int q_pos = POS ? p.q_pos[b] : 0;

    // the group's query rows as the 32-column operand: column t < G is head g * G + t
    u32x4 qf[T::kSteps];
#pragma unroll
    for (int j = 0; j < T::kSteps; ++j) {
      u32x4 x = u32x4{0u, 0u, 0u, 0u};
      if (col < p.G) x = reinterpret_cast<const u32x4*>(p.q)[((long long)b * p.H + (long long)g * p.G + col) * T::kCpr + 2 * j + half];
      qf[j] = x;
    }
    float slope = 0.0f;
    if (POS && p.slopes != nullptr && col < p.G) slope = p.slopes[g * p.G + col] * kLog2e;
    float m_run = -INFINITY, l_run = 0.0f;                    // of head `col` (lanes col < G)
    float acc[GP][kDpl];
#pragma unroll
    for (int i = 0; i < GP; ++i)
#pragma unroll
      for (int e = 0; e < kDpl; ++e) acc[i][e] = 0.0f;

    const int cnt = ta + wave < tb ? (tb - ta - wave + kDecWaves - 1) / kDecWaves : 0;   // this wavefront's tiles
    for (int i0 = 0; i0 < cnt; i0 += 64) {
      const int tile0 = ta + wave + kDecWaves * i0;           // of lane 0; lane j: tile0 + kDecWaves * j
      const int here = cnt - i0 < 64 ? cnt - i0 : 64;
      // ---------------- pages of the next 64 tiles
      int page_a = 0, page_b = 0;
      unsigned int seen = 0xffffffffu;                        // rows of the lane's tile that count (POS)
      {
        const int row0 = (tile0 + kDecWaves * lane) * kTileKeys;
        const bool there = lane < here;
        if (there) page_a = table[row0 >> shift];
        page_b = page_a;
        if (shift == 4 && there && row0 + 16 < rows) page_b = table[(row0 >> 4) + 1];
        const bool bad = page_a < 0 || page_a >= p.n_pages || page_b < 0 || page_b >= p.n_pages;
        if (__ballot(bad) != 0ull) {
          if (lane == 0) s_bad = 1;
          if (bad) page_a = page_b = 0;
        }
        if (POS) {
          const long long at = ((long long)page_a << shift) + (row0 & page_mask);
          const long long bt = shift == 4 ? (long long)page_b << 4 : at + 16;
          seen = 0u;
          if (there) {
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              const int4 x = *reinterpret_cast<const int4*>(p.pos + (c < 4 ? at + 4 * c : bt + 4 * (c - 4)));
              const int y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const unsigned int back = (unsigned int)(q_pos - y[e]);   // a later row: 2^31 and more
                if (back < window && row0 + 4 * c + e < rows) seen |= 1u << (4 * c + e);
              }
            }
          }
        }
      }
      unsigned long long todo = POS ? __ballot(seen != 0u) : (here == 64 ? ~0ull : (1ull << here) - 1ull);
      // place in the pool of the first rows of the two halves of lane j's tile
      auto half_a = [&](int j) -> long long {
        return ((long long)(int)lane_value((unsigned int)page_a, j) << shift) + (((tile0 + kDecWaves * j) * kTileKeys) & page_mask);
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
        const int left = rows - (tile0 + kDecWaves * j) * kTileKeys;
        if (POS || left >= kTileKeys) {
#pragma unroll
          for (int kk = 0; kk < kTileKeys; ++kk)
            dst[kk] = *reinterpret_cast<const VRaw*>((kk < kTileKeys / 2 ? va : vb) + kk * T::kRowBytes + v_lane);
        } else {                                               // rows behind the last one repeat it
#pragma unroll
          for (int kk = 0; kk < kTileKeys; ++kk) {
            const int r = kk < left ? kk : left - 1;
            dst[kk] = *reinterpret_cast<const VRaw*>((r < kTileKeys / 2 ? va : vb) + r * T::kRowBytes + v_lane);
          }
        }
      };

      // Vector-memory operations complete in issue order and the K ring is awaited by count, so the order below is part of the
      // protocol:  K_0, K_1 | V_0 | then per tile i:  K_{i+2}, (positions of i+1,) V_{i+1}
      int j0 = next_tile(), j1 = next_tile(), j2 = next_tile();   // current tile, the next, the one after
      if (j0 >= 0) issue_k(j0, 0);
      if (j1 >= 0) issue_k(j1, 1);
      asm volatile("" ::: "memory");
      VRaw v0[kTileKeys], v1[kTileKeys];
      if (j0 >= 0) load_v(v0, j0);

      auto step = [&](auto par, VRaw (&v_cur)[kTileKeys], VRaw (&v_next)[kTileKeys]) {
        constexpr int PAR = decltype(par)::value;              // ring stage of the current tile
        const int left = rows - (tile0 + kDecWaves * j0) * kTileKeys;   // rows from this tile on (uniform)
        const unsigned int mask = POS ? lane_value(seen, j0) : 0xffffffffu;
        {
          // everything older than this tile's V (32 loads) and, if it was requested, the next K has landed
          if (j1 >= 0) wait_vmcnt<T::kLoads + kTileKeys>(); else wait_vmcnt<kTileKeys>();
          u32x4 kf[T::kSteps];
          frags.template read_at<PAR * T::kTileBytes>(kf);     // in registers on return: the stage is free
          if (j2 >= 0) issue_k(j2, PAR);
          asm volatile("" ::: "memory");
          f32x16 x = {0}, x2 = {0};                            // two chains halve the latency of dependent products
#pragma unroll
          for (int j = 0; j < T::kSteps; j += 2) {
            x = mfma_chunk<DT>(kf[j], qf[j], x);
            x2 = mfma_chunk<DT>(kf[j + 1], qf[j + 1], x2);
          }
          x += x2;                                             // x[v]: row 8*(v/4) + 4*half + v%4, head col
          if (p.cap > 0.0f) {                                  // uniform
#pragma unroll
            for (int v = 0; v < 16; ++v) x[v] = capped(x[v] * p.scale, p.cap, inv_cap) * kLog2e;
          } else {
#pragma unroll
            for (int v = 0; v < 16; ++v) x[v] *= a.c2;
          }
          if (POS) {
            if (p.slopes != nullptr) {                         // uniform
              const long long at = half_a(j0), bt = half_b(j0, at);
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                const int4 y = *reinterpret_cast<const int4*>(p.pos + (c < 2 ? at + 8 * c : bt + 8 * (c - 2)) + 4 * half);
                x[4 * c] -= slope * (float)(q_pos - y.x);
                x[4 * c + 1] -= slope * (float)(q_pos - y.y);
                x[4 * c + 2] -= slope * (float)(q_pos - y.z);
                x[4 * c + 3] -= slope * (float)(q_pos - y.w);
              }
            }
            const unsigned int my = mask >> (4 * half);
#pragma unroll
            for (int v = 0; v < 16; ++v) x[v] = my & (1u << (8 * (v / 4) + v % 4)) ? x[v] : -INFINITY;
          } else if (left < kTileKeys) {                       // a partial tile
            int h4 = 4 * half;
            asm volatile("" : "+v"(h4));                       // keeps this path's temporaries out of the hot loop
#pragma unroll
            for (int v = 0; v < 16; ++v) x[v] = h4 + 8 * (v / 4) + (v % 4) < left ? x[v] : -INFINITY;
          }
          float mt = x[0];
#pragma unroll
          for (int v = 1; v < 16; ++v) mt = fmaxf(mt, x[v]);
          mt = fmaxf(mt, __shfl_xor(mt, 32));
          const float m_new = fmaxf(m_run, mt);
          const float base = m_new == -INFINITY ? 0.0f : m_new;   // logits that are all -inf
          const float alpha = fast_exp2(m_run - base);
          float ls = 0.0f;
          if (col < GP) {
            static_for<16>([&](auto vc) {
              constexpr int v = decltype(vc)::value;
              const float e = fast_exp2(x[v] - base);
              ls += e;
              lds_write32_at<(8 * (v / 4) + (v % 4)) * kPs * 4>(p_mine, e);
            });
            if (half == 0) lds_write32_at<kTileKeys * kPs * 4>(p_col, alpha);
          }
          l_run = l_run * alpha + ls;
          m_run = m_new;
        }
        lds_reads_done();                                      // LDS operations of a wavefront execute in order
        {
          if (j1 >= 0) load_v(v_next, j1);
          asm volatile("" ::: "memory");
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
              if (POS) {                                       // a masked row may hold anything
                const bool take = (mask >> (k4 + kk)) & 1u;    // uniform
#pragma unroll
                for (int e = 0; e < kDpl; ++e) vx[e] = take ? vx[e] : 0.0f;
              }
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

    // ---------------- merge the wavefronts
    l_run += __shfl_xor(l_run, 32);
    if (lane < GP) {
      s_m[wave][lane] = m_run;
      s_l[wave][lane] = l_run;
    }
    __syncthreads();                                          // every wavefront is done with its ring
    float (*s_acc)[GP][D] = reinterpret_cast<float (*)[GP][D]>(&s_tile[0][0][0]);
#pragma unroll
    for (int i = 0; i < GP; ++i)
#pragma unroll
      for (int e = 0; e < kDpl; ++e) s_acc[wave][i][lane * kDpl + e] = acc[i][e];
    __syncthreads();
    const bool bad = s_bad != 0;
    const bool whole = ta == 0 && tb == tiles;
    const long long slot = ta > 0 ? 2 * (long long)blockIdx.x : 2 * (long long)blockIdx.x + 1;
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
      if (bad) L = NAN;                                       // a page that is not in the pool: the head's result is none
      if (!whole) {
        st_dev_f2(reinterpret_cast<float2*>(a.part_acc + slot * GP * D + idx), sum.x, sum.y);
        if (e == 0) st_dev_f2(&a.part_ml[slot * GP + i], M, L);
      } else if (i < p.G) {
        const long long row = (long long)b * p.H + (long long)g * p.G + i;
        const bool none = L == 0.0f;                          // every row masked
        p.out[row * D + e] = none ? 0.0f : sum.x / L;
        p.out[row * D + e + 1] = none ? 0.0f : sum.y / L;
        if (p.lse != nullptr && e == 0) p.lse[row] = none ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
      }
    }
    if (!whole) {
      // ---------------- publish the part; merge the head if all its parts are published
      drain_vmem();
      __syncthreads();                                        // every thread's share of the part is visible to the device
      const long long w0 = uniform64(quotient(head_start, share));
      const int parts = (int)(uniform64(quotient(head_start + tiles - 1, share)) - w0) + 1;
      if (wave == 0) {
        if (lane == 0) {
          st_dev(&a.flags[slot], a.tag);
          drain_vmem();
        }
        bool all = true;
        for (int i = lane; i < parts; i += 64) all &= ld_dev(&a.flags[part_slot(w0, i)]) == a.tag;
        const bool every = __ballot(!all) == 0ull;
        if (lane == 0) s_flag = every ? 1 : 0;
      }
      __syncthreads();
      if (s_flag != 0) {
        for (int i = threadIdx.x; i < parts; i += kDecThreads) st_dev(&a.flags[part_slot(w0, i)], 0ull);
        static_assert(sizeof(s_tile) >= kPartChunk * GP * sizeof(float2), "the ring is the merge's buffer");
        merge_parts<D, GP>(a, b, g, w0, parts, reinterpret_cast<float2 (*)[GP]>(&s_tile[0][0][0]));
      }
    }
    __syncthreads();                                          // the ring, s_m and s_bad are free again
    if (threadIdx.x == 0) s_bad = 0;
    t = head_start + tb;
    head_start += tiles;
    ++hb;
    __syncthreads();
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

template <int DT, int D, int GP, bool POS>
int32_t launch_one(const PagedArgs& a, hipStream_t s) {
  static const int wgs = resident(paged_decode_kernel<DT, D, GP, POS>);
  ProfScope ps(KID_PAGED_DECODE, s);
  hipLaunchKernelGGL((paged_decode_kernel<DT, D, GP, POS>), dim3((unsigned)wgs), dim3(kDecThreads), 0, s, a);
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
#define LAVA_PAGED_CASE(DT, D, GP) \
  if (d.dtype == DT && d.head_dim == D && gp == GP)        \
    return p.pos != nullptr ? launch_one<DT, D, GP, true>(a, s) : launch_one<DT, D, GP, false>(a, s);
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
