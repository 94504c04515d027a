// Rotary positions: pairs of a head's leading values turned by position * frequency, keys and values written to the slots
// of the paged cache on the way.
//
// An angle is a 64-bit fraction of a turn: position * turns modulo 2^64 is exact, so that position 10^6 is as accurate as
// position 1.  Its two leading bits (after rounding) are the quadrant, the rest an angle of at most pi / 4 whose sine
// and cosine are Taylor sums (their next terms are 2e-9 and 1e-10 there).  A token's sines and cosines are formed once, by
// one lane each, and serve all of its heads through LDS.
//
// A unit of work is 32 bytes of a head: the E = 16 / elem pairs j E .. j E + E - 1, which are two chunks of 16 bytes half
// a rotation apart (or, interleaved, next to each other); behind the rotated part two neighbouring chunks that pass.
// Bound by HBM: every row is read and written once.  8197 tokens of 32 + 2 x 8 heads (202 MB): 42 us, 4.8 TB/s, where a copy takes
// 40.5; 4115 x 32 heads of 32-bit values, head by head: 26.6 us, 5.1 TB/s (27.4 without the row ahead).  64 tokens: 3.5 us.
#include "common.h"
#include "tile_ring.h"

namespace lava {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotMaxPairs = 64;

// (cos, sin) of a fraction of a turn.
__device__ __forceinline__ float2 unit_turn(unsigned long long phase) {
  const unsigned int hi = (unsigned int)(phase >> 32);
  const unsigned int quad = (hi + 0x20000000u) >> 30;              // nearest quarter turn
  const int rest = (int)(hi - (quad << 30));                       // in 2^-32 turns, |rest| <= 2^29
  const float x = (float)rest * 1.4629180792671596e-9f;            // 2 pi / 2^32
  const float y = x * x;
  float s = fmaf(y, 2.7557319e-6f, -1.9841270e-4f);                // x^9 / 9!, -x^7 / 7!
  s = fmaf(y, s, 8.3333333e-3f);
  s = fmaf(y, s, -1.6666667e-1f);
  s = fmaf(x * y, s, x);
  float c = fmaf(y, -2.7557319e-7f, 2.4801587e-5f);                // -x^10 / 10!, x^8 / 8!
  c = fmaf(y, c, -1.3888889e-3f);
  c = fmaf(y, c, 4.1666667e-2f);
  c = fmaf(y, c, -0.5f);
  c = fmaf(y, c, 1.0f);
  const float a = quad & 1u ? s : c, b = quad & 1u ? c : s;        // a quarter turn: (c, s) -> (-s, c)
  return make_float2((quad + 1u) & 2u ? -a : a, quad & 2u ? -b : b);
}

// The pairs of one unit, turned.  a, b: the two chunks; cs[i]: cosine and sine of pair i; n: pairs that are turned, the
// others keep their bits.
template <int DT>
__device__ __forceinline__ void turn_halves(u32x4& a, u32x4& b, const float2* cs) {
  if constexpr (DT == LAVA_BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = cs[2 * i], q = cs[2 * i + 1];
      const float a0 = bf16_low(a[i]), a1 = bf16_high(a[i]), b0 = bf16_low(b[i]), b1 = bf16_high(b[i]);
      a[i] = pack_bf16(a0 * p.x - b0 * p.y, a1 * q.x - b1 * q.y);
      b[i] = pack_bf16(a0 * p.y + b0 * p.x, a1 * q.y + b1 * q.x);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = cs[i];
      const float a0 = __uint_as_float(a[i]), b0 = __uint_as_float(b[i]);
      a[i] = __float_as_uint(a0 * p.x - b0 * p.y);
      b[i] = __float_as_uint(a0 * p.y + b0 * p.x);
    }
  }
}

template <int DT>
__device__ __forceinline__ void turn_neighbours(u32x4& a, u32x4& b, const float2* cs, int n) {
  u32x4* half[2] = {&a, &b};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    u32x4& x = *half[h];
    if constexpr (DT == LAVA_BF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {                                // a dword is a pair
        const float2 p = cs[4 * h + i];
        const float x0 = bf16_low(x[i]), x1 = bf16_high(x[i]);
        const unsigned int y = pack_bf16(x0 * p.x - x1 * p.y, x0 * p.y + x1 * p.x);
        x[i] = 4 * h + i < n ? y : x[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 p = cs[2 * h + i];
        const float x0 = __uint_as_float(x[2 * i]), x1 = __uint_as_float(x[2 * i + 1]);
        const bool mine = 2 * h + i < n;
        x[2 * i] = mine ? __float_as_uint(x0 * p.x - x1 * p.y) : x[2 * i];
        x[2 * i + 1] = mine ? __float_as_uint(x0 * p.y + x1 * p.x) : x[2 * i + 1];
      }
    }
  }
}

// Halves whose length is no multiple of a chunk: value by value, pair p by whoever has unit p / E, the values behind the
// rotated part spread over the units.  8197 tokens of 32 + 2 x 8 heads, 38 values of 128 turned: 130 us, where whole chunks take 40.
template <int DT, int D>
__device__ __forceinline__ void turn_values(const char* src, char* dst, int j, int rot, const float2* cs) {
  constexpr int E = 16 / Elem<DT>::kBytes, kUnits = D / E / 2;
  const int half = rot / 2;
  if constexpr (DT == LAVA_BF16) {
    const unsigned short* x = reinterpret_cast<const unsigned short*>(src);
    unsigned short* y = reinterpret_cast<unsigned short*>(dst);
    for (int p = j * E; p < (j + 1) * E && p < half; ++p) {
      const float a = bf16_low(x[p]), b = bf16_low(x[p + half]);
      const float2 t = cs[p];
      const unsigned int r = pack_bf16(a * t.x - b * t.y, a * t.y + b * t.x);
      y[p] = (unsigned short)(r & 0xffffu);
      y[p + half] = (unsigned short)(r >> 16);
    }
    for (int e = rot + j; e < D; e += kUnits) y[e] = x[e];
  } else {
    const float* x = reinterpret_cast<const float*>(src);
    float* y = reinterpret_cast<float*>(dst);
    for (int p = j * E; p < (j + 1) * E && p < half; ++p) {
      const float a = x[p], b = x[p + half];
      const float2 t = cs[p];
      y[p] = a * t.x - b * t.y;
      y[p + half] = a * t.y + b * t.x;
    }
    const unsigned int* xb = reinterpret_cast<const unsigned int*>(src);
    unsigned int* yb = reinterpret_cast<unsigned int*>(dst);
    for (int e = rot + j; e < D; e += kUnits) yb[e] = xb[e];
  }
}

// A workgroup a token.
template <int DT, int D>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const RotaryArgs a) {
  constexpr int E = 16 / Elem<DT>::kBytes;                           // values of a chunk = pairs of a unit
  constexpr int kUnits = D / E / 2;                                // units of a head
  constexpr int kRowBytes = D * Elem<DT>::kBytes;
  __shared__ float2 s_cs[kRotMaxPairs];
  const long long token = blockIdx.x;
  const int pairs = a.rot / 2, pos = a.positions[token];
  const int rows = a.hq + 2 * a.hkv;                               // of a token: heads to turn into `out`, keys, values
  const bool by_value = a.interleaved == 0 && pairs % E != 0;      // uniform
  const int turned = a.interleaved ? (pairs + E - 1) / E : pairs / E;   // units with turned pairs
  const int j = threadIdx.x % kUnits;
  // chunks of this thread's unit
  const bool apart = !a.interleaved && j < turned;
  const int c0 = apart ? j : 2 * j, c1 = apart ? j + turned : 2 * j + 1;

  // one row ahead: where it lies and, unless it goes value by value, its chunks
  const char* src = nullptr;
  char* dst = nullptr;                                             // null: the row has no slot
  bool turn = true;
  u32x4 x0, x1;
  auto fetch = [&](int row) {
    dst = nullptr;
    if (row >= rows) return;
    if (row < a.hq) {
      turn = true;
      src = a.x + token * a.x_token + row * a.x_head;
      dst = a.out + token * a.out_token + row * a.out_head;
    } else {
      turn = row - a.hq < a.hkv;
      const int g = turn ? row - a.hq : row - a.hq - a.hkv;
      const long long slot = a.slots[token * a.hkv + g];
      if (slot < 0 || slot >= a.pool_rows) return;
      src = turn ? a.k + token * a.k_token + g * kRowBytes : a.v + token * a.v_token + g * kRowBytes;
      dst = (turn ? a.k_pages : a.v_pages) + slot * kRowBytes;
      if (turn && j == 0 && pos >= 0 && a.pos_pages != nullptr) a.pos_pages[slot] = pos;
    }
    if (turn && by_value) return;
    x0 = *reinterpret_cast<const u32x4*>(src + c0 * 16);
    x1 = *reinterpret_cast<const u32x4*>(src + c1 * 16);
  };
  int row = threadIdx.x / kUnits;
  fetch(row);
  if ((int)threadIdx.x < pairs) {
    const float2 cs = unit_turn((unsigned long long)(unsigned int)pos * a.turns[threadIdx.x]);
    s_cs[threadIdx.x] = make_float2(cs.x * a.cos_mul, cs.y * a.sin_mul);
  }
  __syncthreads();
  if (pos < 0) return;                                             // uniform: the token is left out
  for (; row < rows; ) {
    if (dst != nullptr) {
      if (turn && by_value) {
        turn_values<DT, D>(src, dst, j, a.rot, s_cs);
      } else {
        if (turn && j < turned) {
          if (a.interleaved) turn_neighbours<DT>(x0, x1, &s_cs[j * E], pairs - j * E);
          else turn_halves<DT>(x0, x1, &s_cs[j * E]);
        }
        *reinterpret_cast<u32x4*>(dst + c0 * 16) = x0;
        *reinterpret_cast<u32x4*>(dst + c1 * 16) = x1;
      }
    }
    row += kRotThreads / kUnits;
    fetch(row);
  }
}

template <int DT, int D>
int32_t launch_rotary_type(const RotaryArgs& a, hipStream_t s) {
  ProfScope ps(KID_ROTARY, s);
  constexpr long long kTokens = 1ll << 23;                           // a launch's threads are counted in 32 bits
  for (long long t0 = 0; t0 < a.n_tokens; t0 += kTokens) {
    RotaryArgs b = a;
    b.n_tokens = a.n_tokens - t0 < kTokens ? a.n_tokens - t0 : kTokens;
    b.positions += t0;
    if (a.x != nullptr) {
      b.x += t0 * a.x_token;
      b.out += t0 * a.out_token;
    }
    if (a.slots != nullptr) {
      b.k += t0 * a.k_token;
      b.v += t0 * a.v_token;
      b.slots += t0 * a.hkv;
    }
    hipLaunchKernelGGL((rotary_kernel<DT, D>), dim3((unsigned)b.n_tokens), dim3(kRotThreads), 0, s, b);
    const int32_t st = launch_status();
    if (st != LAVA_OK) return st;
  }
  return LAVA_OK;
}

}  // namespace

int32_t launch_rotary(const RotaryArgs& a, int32_t dtype, int32_t head_dim, hipStream_t s) {
  if (dtype == LAVA_BF16)
    return head_dim == 128 ? launch_rotary_type<LAVA_BF16, 128>(a, s) : launch_rotary_type<LAVA_BF16, 64>(a, s);
  return head_dim == 128 ? launch_rotary_type<LAVA_F32, 128>(a, s) : launch_rotary_type<LAVA_F32, 64>(a, s);
}

}  // namespace lava
