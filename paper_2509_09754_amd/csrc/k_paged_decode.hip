// Decode-step attention over the pages of the paged cache.
//
// One workgroup per head of a sequence; its wavefronts take the head's rows in turn, a lane owns d_h / 64 columns, the logits
// are sums over the wavefront, the softmax is online per wavefront and the wavefronts are merged at the end.
#include <math.h>

#include "common.h"
#include "tile_ring.h"

namespace lava {

namespace {

constexpr int kWaves = 4;

template <int DT, int D, int GP>
__global__ void __launch_bounds__(kWaves * 64) paged_decode_kernel(const PagedDecodeArgs a) {
  constexpr int kDpl = D / 64, kRowBytes = D * Elem<DT>::kBytes;
  __shared__ float s_acc[kWaves][GP][D], s_m[kWaves][GP], s_l[kWaves][GP];
  __shared__ int s_bad;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int hb = blockIdx.x, b = hb / a.H_kv, g = hb - b * a.H_kv;
  const int rows = a.head_rows[hb];
  if (threadIdx.x == 0) s_bad = rows < 0 || rows > (long long)a.max_blocks << a.page_shift ? 1 : 0;
  __syncthreads();
  auto value = [&](const char* row, int e) -> float {
    if constexpr (DT == LAVA_BF16) return bf16_low(reinterpret_cast<const unsigned short*>(row)[e]);
    else return reinterpret_cast<const float*>(row)[e];
  };
  float q[GP][kDpl], acc[GP][kDpl], m[GP], l[GP];
#pragma unroll
  for (int t = 0; t < GP; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.0f;
#pragma unroll
    for (int e = 0; e < kDpl; ++e) {
      acc[t][e] = 0.0f;
      q[t][e] = t < a.G ? value(a.q + ((long long)b * a.H + g * a.G + t) * kRowBytes, lane * kDpl + e) : 0.0f;
    }
  }
  const int n = s_bad ? 0 : rows;
  for (int r = wave; r < n; r += kWaves) {
    const long long page = a.block_table[(long long)hb * a.max_blocks + (r >> a.page_shift)];
    if (page < 0 || page >= a.n_pages) {
      if (lane == 0) s_bad = 1;
      continue;
    }
    const long long slot = (page << a.page_shift) + (r & ((1 << a.page_shift) - 1));
    int back = 0;
    if (a.pos != nullptr) {
      back = a.q_pos[b] - a.pos[slot];
      if (back < 0 || (a.window > 0 && back >= a.window)) continue;
    }
    const char* k = a.k + slot * kRowBytes;
    const char* v = a.v + slot * kRowBytes;
    float kx[kDpl], vx[kDpl];
#pragma unroll
    for (int e = 0; e < kDpl; ++e) {
      kx[e] = value(k, lane * kDpl + e);
      vx[e] = value(v, lane * kDpl + e);
    }
#pragma unroll
    for (int t = 0; t < GP; ++t) {
      float z = 0.0f;
#pragma unroll
      for (int e = 0; e < kDpl; ++e) z = fmaf(q[t][e], kx[e], z);
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) z += __shfl_xor(z, d);
      z *= a.scale;
      if (a.cap > 0.0f) z = a.cap * tanhf(z / a.cap);
      if (a.slopes != nullptr && t < a.G) z -= a.slopes[g * a.G + t] * (float)back;
      const float mn = fmaxf(m[t], z);
      const float base = mn == -INFINITY ? 0.0f : mn, keep = expf(m[t] - base), p = expf(z - base);
      l[t] = l[t] * keep + p;
      m[t] = mn;
#pragma unroll
      for (int e = 0; e < kDpl; ++e) acc[t][e] = acc[t][e] * keep + p * vx[e];
    }
  }
#pragma unroll
  for (int t = 0; t < GP; ++t) {
    if (lane == 0) {
      s_m[wave][t] = m[t];
      s_l[wave][t] = l[t];
    }
#pragma unroll
    for (int e = 0; e < kDpl; ++e) s_acc[wave][t][lane * kDpl + e] = acc[t][e];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.G * D; i += kWaves * 64) {
    const int t = i / D, e = i % D;
    float M = -INFINITY, L = 0.0f, sum = 0.0f;
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_m[w][t]);
    for (int w = 0; w < kWaves; ++w) {
      const float f = M == -INFINITY ? 0.0f : expf(s_m[w][t] - M);
      L += f * s_l[w][t];
      sum += f * s_acc[w][t][e];
    }
    const long long row = (long long)b * a.H + g * a.G + t;
    a.out[row * D + e] = s_bad ? NAN : L == 0.0f ? 0.0f : sum / L;
    if (e == 0 && a.lse != nullptr) a.lse[row] = s_bad ? NAN : L == 0.0f ? -INFINITY : M + logf(L);
  }
}

template <int DT, int D, int GP>
int32_t launch_one(const PagedDecodeArgs& a, hipStream_t s) {
  ProfScope ps(KID_PAGED_DECODE, s);
  hipLaunchKernelGGL((paged_decode_kernel<DT, D, GP>), dim3((unsigned)(a.batch * a.H_kv)), dim3(kWaves * 64), 0, s, a);
  return launch_status();
}

}  // namespace

size_t paged_decode_bytes(const lava_layer_desc&) { return 256; }

int32_t launch_paged_decode(const lava_layer_desc& d, const PagedDecodeArgs& a, void*, hipStream_t s) {
  const int gp = a.G <= 1 ? 1 : a.G <= 2 ? 2 : a.G <= 4 ? 4 : 8;
#define LAVA_PAGED_CASE(DT, D, GP) if (d.dtype == DT && d.head_dim == D && gp == GP) return launch_one<DT, D, GP>(a, s);
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
