// One step of beam search: c = score + (x - log sum exp x) of every beam and token, and the best n_out of a group of beams.
//
// Which of two candidates is better is a comparison across beams, so the sums of exponentials decide it: c is formed in 64 bits.  Inside
// a beam candidates are in the order of their logits, which is exact, so of each beam the best n_out logits suffice.
//   rows   a workgroup per 8192 tokens of a beam, held in registers: maximum, sum of exponentials (64 bits), and the best n_out of
//          them.  The n_out-th largest of a wavefront's 64 lane maxima is a bound below which no token counts; what is not below the
//          highest of these bounds is listed (a few dozen tokens as a rule) and ranked by counting.
//   pick   a workgroup per group of beams: sums over the parts in order, candidates of all parts, ranked the same way.
// Which thread holds which token does not depend on where the row begins, so equal rows have equal sums, bit for bit.
//
// Exponentials: 2^y = 2^rint(y) p(y - rint(y)), p the Taylor polynomial of 2^f of degree 10, |f| <= 1/2: left out is less than
// (ln 2 / 2)^11 / 11! < 3e-13 of it.  14 64-bit instructions a token, at the rate of 32-bit ones on this device.
#include "common.h"
#include "decode_parts.h"
#include "tile_ring.h"

namespace lava {

namespace {

constexpr int kBeamThreads = 256, kBeamWaves = kBeamThreads / 64;
constexpr int kPart = 8192;                    // tokens of a part
constexpr int kPer = kPart / kBeamThreads;     // tokens a thread holds
constexpr int kListed = 1024;                  // candidates that are ranked by counting

struct BeamKernelArgs {
  BeamArgs b;
  int parts;                                   // of a row
  double* sum;                                 // [rows][parts] sum of exp(x - maximum); NaN: the beam has no continuation
  float* top;                                  // [rows][parts] maximum
  unsigned long long* best;                    // [rows][parts][n_out] keys, the best first; 0: none
};

// Larger logit first, then the smaller token; 0 is nothing.  -0 and +0 are equal.
__device__ __forceinline__ unsigned long long token_key(float x, unsigned int token) {
  return ((unsigned long long)score_key(x) << 32) | (0xffffffffu - token);
}
__device__ __forceinline__ float key_logit(unsigned long long key) {
  const unsigned int u = (unsigned int)(key >> 32);
  return __uint_as_float((u & 0x80000000u) != 0u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ unsigned int key_token(unsigned long long key) { return 0xffffffffu - (unsigned int)key; }

// 2^y for y <= 0 (smaller than -1100: zero).
__device__ __forceinline__ double exp2_of(double y) {
  y = y > -1100.0 ? y : -1100.0;
  const double n = __builtin_rint(y), f = y - n;
  double p = 7.0549116208011232e-9;            // (ln 2)^10 / 10!
  p = fma(p, f, 1.0178086009239699e-7);
  p = fma(p, f, 1.3215486790144309e-6);
  p = fma(p, f, 1.5252733804059840e-5);
  p = fma(p, f, 1.5403530393381609e-4);
  p = fma(p, f, 1.3333558146428443e-3);
  p = fma(p, f, 9.6181291076284771e-3);
  p = fma(p, f, 5.5504108664821580e-2);
  p = fma(p, f, 2.4022650695910071e-1);
  p = fma(p, f, 6.9314718055994531e-1);
  p = fma(p, f, 1.0);
  return __builtin_ldexp(p, (int)n);
}
constexpr double kLog2e64 = 1.4426950408889634074;

struct alignas(2) Bf16x8 { unsigned short x[8]; };
struct alignas(4) F32x4 { float x[4]; };

// Is beam `row` one whose logits count?
__device__ __forceinline__ bool is_live(const BeamArgs& b, int row) {
  return isfinite(b.scores[row]) && (b.done == nullptr || b.done[row] == 0);
}

// The `count`-th largest of the lanes' values.
__device__ __forceinline__ unsigned int nth_of_wave(unsigned int x, int count) {
  const int lane = threadIdx.x & 63;
  int before = 0;
#pragma unroll
  for (int l = 0; l < 64; ++l) {
    const unsigned int y = lane_value(x, l);
    before += y > x || (y == x && l < lane) ? 1 : 0;
  }
  const unsigned long long at = __ballot(before == count - 1);
  return lane_value(x, __builtin_ctzll(at));
}

__device__ __forceinline__ unsigned long long max_key_of_wave(unsigned long long x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const unsigned long long y = __shfl_xor(x, m);
    x = y > x ? y : x;
  }
  return x;
}

template <int DT>
__global__ void __launch_bounds__(kBeamThreads) beam_rows_kernel(const BeamKernelArgs a) {
  __shared__ unsigned long long s_list[kListed];
  __shared__ double s_sum[kBeamWaves];
  __shared__ unsigned long long s_key[kBeamWaves];
  __shared__ unsigned int s_top[kBeamWaves], s_bound[kBeamWaves], s_bad[kBeamWaves];
  __shared__ int s_count;
  const BeamArgs& b = a.b;
  const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (!is_live(b, row)) return;                                // uniform
  constexpr int kVec = DT == LAVA_BF16 ? 8 : 4, kLoads = kPer / kVec;   // tokens of a load: thread t has tokens t * kVec .. of each kVec * 256
  const char* from = b.logits + (long long)row * b.stride_bytes;
  const long long first = (long long)part * kPart;
  const int here = b.vocab - first < kPart ? (int)(b.vocab - first) : kPart;
  float x[kPer];
#pragma unroll
  for (int l = 0; l < kLoads; ++l) {
    const int at = l * kVec * kBeamThreads + (int)threadIdx.x * kVec;
    const char* src = from + (first + at) * Elem<DT>::kBytes;
    if (at + kVec <= here) {
      if constexpr (DT == LAVA_BF16) {
        const Bf16x8 r = *reinterpret_cast<const Bf16x8*>(src);
#pragma unroll
        for (int e = 0; e < kVec; ++e) x[l * kVec + e] = __uint_as_float((unsigned int)r.x[e] << 16);
      } else {
        const F32x4 r = *reinterpret_cast<const F32x4*>(src);
#pragma unroll
        for (int e = 0; e < kVec; ++e) x[l * kVec + e] = r.x[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        float y = -INFINITY;
        if (at + e < here)
          y = DT == LAVA_BF16 ? __uint_as_float((unsigned int)reinterpret_cast<const unsigned short*>(src)[e] << 16)
                              : reinterpret_cast<const float*>(src)[e];
        x[l * kVec + e] = y;
      }
    }
  }
  auto token_of = [&](int i) { return (unsigned int)first + (unsigned int)((i / kVec) * kVec * kBeamThreads + (int)threadIdx.x * kVec + i % kVec); };
  // maximum, bound, NaN and +inf
  float most = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    bad |= !(x[i] < INFINITY);
    most = fmaxf(most, x[i]);
  }
  const unsigned int mine = most == -INFINITY ? 0u : score_key(most);
  const unsigned int bound = nth_of_wave(mine, b.n_out);
  unsigned int top = mine;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const unsigned int y = (unsigned int)__shfl_xor((int)top, m);
    top = y > top ? y : top;
  }
  const bool any_bad = __ballot(bad) != 0ull;
  if (lane == 0) {
    s_top[wave] = top;
    s_bound[wave] = bound;
    s_bad[wave] = any_bad ? 1u : 0u;
  }
  if (threadIdx.x == 0) s_count = 0;
  __syncthreads();
  unsigned int limit = s_bound[0], wrong = s_bad[0];
  top = s_top[0];
#pragma unroll
  for (int w = 1; w < kBeamWaves; ++w) {
    limit = s_bound[w] > limit ? s_bound[w] : limit;
    top = s_top[w] > top ? s_top[w] : top;
    wrong |= s_bad[w];
  }
  limit = limit == 0u ? 1u : limit;                            // nothing is no candidate
  const long long out = (long long)row * a.parts + part;
  if (wrong != 0u || top == 0u) {                              // uniform
    if (threadIdx.x == 0) {
      a.sum[out] = wrong != 0u ? NAN : 0.0;
      a.top[out] = -INFINITY;
    }
    if ((int)threadIdx.x < b.n_out) a.best[out * b.n_out + threadIdx.x] = 0ull;
    return;
  }
  const float m = key_logit((unsigned long long)top << 32);
  const double most64 = (double)m;                             // the difference first: m log2 e may be too large for its last bits to count
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) sum += exp2_of(((double)x[i] - most64) * kLog2e64);
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) sum += __shfl_xor(sum, s);
  if (lane == 0) s_sum[wave] = sum;
  // the list
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const bool in = x[i] > -INFINITY && score_key(x[i]) >= limit;
    const unsigned long long who = __ballot(in);
    if (who == 0ull) continue;
    int at = 0;
    if (lane == 0) at = atomicAdd(&s_count, __popcll(who));
    at = (int)lane_value((unsigned int)at, 0) + __popcll(who & ((1ull << lane) - 1ull));
    if (in && at < kListed) s_list[at] = token_key(x[i], token_of(i));
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double all = s_sum[0];
#pragma unroll
    for (int w = 1; w < kBeamWaves; ++w) all += s_sum[w];
    a.sum[out] = all;
    a.top[out] = m;
  }
  const int count = s_count;
  unsigned long long* best = a.best + out * b.n_out;
  if (count <= kListed) {
    for (int i = threadIdx.x; i < count; i += kBeamThreads) {
      const unsigned long long key = s_list[i];
      int rank = 0;
      for (int j = 0; j < count; ++j) rank += s_list[j] > key ? 1 : 0;
      if (rank < b.n_out) best[rank] = key;
    }
    for (int i = count + (int)threadIdx.x; i < b.n_out; i += kBeamThreads) best[i] = 0ull;
    return;
  }
  // more equals than the list holds: the best one by one
  unsigned long long last = ~0ull;
  for (int k = 0; k < b.n_out; ++k) {
    unsigned long long key = 0ull;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const unsigned long long y = x[i] > -INFINITY ? token_key(x[i], token_of(i)) : 0ull;
      key = y < last && y > key ? y : key;
    }
    key = max_key_of_wave(key);
    if (lane == 0) s_key[wave] = key;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kBeamWaves; ++w) key = s_key[w] > key ? s_key[w] : key;
    __syncthreads();
    if (threadIdx.x == 0) best[k] = key;
    last = key;
  }
}

// A candidate: c in an order-preserving map to integers (0: none), then what decides between equals: the beam, the logit, the token.
struct Candidate {
  unsigned long long c, key;
  int beam;
};
__device__ __forceinline__ unsigned long long order_of(double c) {
  const unsigned long long u = (unsigned long long)__double_as_longlong(c + 0.0);
  return u ^ ((unsigned long long)((long long)u >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ double value_of(unsigned long long u) {
  return __longlong_as_double((long long)((u >> 63) != 0ull ? u ^ 0x8000000000000000ull : ~u));
}
__device__ __forceinline__ bool before(const Candidate& x, const Candidate& y) {
  if (x.c != y.c) return x.c > y.c;
  if (x.beam != y.beam) return x.beam < y.beam;
  return x.key > y.key;
}

constexpr int kMostBeams = 64;
__global__ void __launch_bounds__(kBeamThreads) beam_pick_kernel(const BeamKernelArgs a) {
  __shared__ Candidate s_list[kListed];
  __shared__ double s_base[kMostBeams];                        // log sum exp; NaN: no continuation
  __shared__ float s_score[kMostBeams];                        // read once: scores_out may be the same buffer
  __shared__ Candidate s_best[kBeamWaves];
  __shared__ unsigned int s_bound[kBeamWaves];
  __shared__ int s_over[kMostBeams], s_count;
  const BeamArgs& b = a.b;
  const int group = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int i = wave; i < b.beams; i += kBeamWaves) {
    const int row = group * b.beams + i;
    const float score = b.scores[row];
    const bool over = b.done != nullptr && b.done[row] != 0;
    double base = NAN;
    if (isfinite(score) && !over) {                            // uniform
      float m = -INFINITY;
      for (int q = lane; q < a.parts; q += 64) m = fmaxf(m, a.top[(long long)row * a.parts + q]);
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
      double sum = 0.0;
      for (int q = lane; q < a.parts; q += 64) {
        const float t = a.top[(long long)row * a.parts + q];
        const double z = a.sum[(long long)row * a.parts + q];
        sum += isnan(z) ? z : t == -INFINITY ? 0.0 : z * exp2_of(((double)t - (double)m) * kLog2e64);
      }
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) sum += __shfl_xor(sum, s);
      if (sum > 0.0) base = (double)m + log(sum);              // a NaN is not
    } else if (isfinite(score) && over) {
      base = 0.0;
    }
    if (lane == 0) {
      s_base[i] = base;
      s_over[i] = over ? 1 : 0;
      s_score[i] = score;
    }
  }
  if (threadIdx.x == 0) s_count = 0;
  __syncthreads();
  const int each = a.parts * b.n_out, all = b.beams * each;
  auto candidate = [&](int i) {
    Candidate r = {0ull, 0ull, i / each};
    const int j = i - r.beam * each, row = group * b.beams + r.beam;
    const double base = s_base[r.beam];
    if (isnan(base)) return r;
    const double score = (double)s_score[r.beam];
    if (s_over[r.beam] != 0) {
      if (j != 0) return r;
      r.c = order_of(score);
      r.key = token_key(0.0f, (unsigned int)b.pad_token);
      return r;
    }
    r.key = a.best[(long long)row * each + j];
    if (r.key != 0ull) r.c = order_of(score + ((double)key_logit(r.key) - base));
    return r;
  };
  unsigned int mine = 0u;
  for (int i = threadIdx.x; i < all; i += kBeamThreads) {
    const unsigned int top = (unsigned int)(candidate(i).c >> 32);
    mine = top > mine ? top : mine;
  }
  const unsigned int bound = nth_of_wave(mine, b.n_out);
  if (lane == 0) s_bound[wave] = bound;
  __syncthreads();
  unsigned int limit = s_bound[0];
#pragma unroll
  for (int w = 1; w < kBeamWaves; ++w) limit = s_bound[w] > limit ? s_bound[w] : limit;
  for (int i = threadIdx.x; i < all; i += kBeamThreads) {
    const Candidate r = candidate(i);
    if (r.c == 0ull || (unsigned int)(r.c >> 32) < limit) continue;
    const int at = atomicAdd(&s_count, 1);
    if (at < kListed) s_list[at] = r;
  }
  __syncthreads();
  const int count = s_count;
  auto write = [&](int k, const Candidate& r) {
    const bool none = r.c == 0ull;
    const int row = none ? -1 : group * b.beams + r.beam, at = group * b.n_out + k;
    const int token = none ? -1 : (int)key_token(r.key);
    b.parents[at] = row;
    b.tokens[at] = token;
    b.scores_out[at] = none ? -INFINITY : (float)value_of(r.c);
    if (b.done_out != nullptr) b.done_out[at] = none || s_over[r.beam] != 0 || token == b.end_token ? 1 : 0;
    for (int t = 0; t < b.n_tables; ++t)
      b.sources[(long long)t * b.batch * b.n_out + at] = none ? -1 : row + t * b.batch * b.beams;
  };
  if (count <= kListed) {
    for (int i = threadIdx.x; i < count; i += kBeamThreads) {
      const Candidate r = s_list[i];
      int rank = 0;
      for (int j = 0; j < count; ++j) rank += before(s_list[j], r) ? 1 : 0;
      if (rank < b.n_out) write(rank, r);
    }
    for (int i = count + (int)threadIdx.x; i < b.n_out; i += kBeamThreads) write(i, Candidate{0ull, 0ull, 0});
    return;
  }
  Candidate last = {~0ull, ~0ull, -1};
  for (int k = 0; k < b.n_out; ++k) {
    Candidate r = {0ull, 0ull, 0};
    for (int i = threadIdx.x; i < all; i += kBeamThreads) {
      const Candidate y = candidate(i);
      if (y.c != 0ull && before(last, y) && before(y, r)) r = y;
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const Candidate y = {__shfl_xor(r.c, s), __shfl_xor(r.key, s), __shfl_xor(r.beam, s)};
      if (before(y, r)) r = y;
    }
    if (lane == 0) s_best[wave] = r;
    __syncthreads();
    for (int w = 0; w < kBeamWaves; ++w)
      if (before(s_best[w], r)) r = s_best[w];
    __syncthreads();
    if (threadIdx.x == 0) write(k, r);
    last = r;
  }
}

int parts_of(int64_t vocab) { return (int)((vocab + kPart - 1) / kPart); }

struct BeamLayout {
  size_t off_top, off_best, bytes;
};
BeamLayout beam_layout(int32_t batch, int32_t beams, int64_t vocab, int32_t n_out) {
  const size_t n = (size_t)batch * beams * parts_of(vocab);
  BeamLayout l;
  l.off_top = align_up(n * sizeof(double));
  l.off_best = l.off_top + align_up(n * sizeof(float));
  l.bytes = l.off_best + align_up(n * n_out * sizeof(unsigned long long));
  return l;
}

}  // namespace

size_t beam_step_bytes(int32_t batch, int32_t beams, int64_t vocab, int32_t n_out) { return beam_layout(batch, beams, vocab, n_out).bytes; }

int32_t launch_beam_step(const BeamArgs& b, int32_t dtype, void* ws, hipStream_t s) {
  BeamKernelArgs a;
  a.b = b;
  a.parts = parts_of(b.vocab);
  const BeamLayout l = beam_layout(b.batch, b.beams, b.vocab, b.n_out);
  a.sum = static_cast<double*>(ws);
  a.top = reinterpret_cast<float*>(static_cast<char*>(ws) + l.off_top);
  a.best = reinterpret_cast<unsigned long long*>(static_cast<char*>(ws) + l.off_best);
  const unsigned wgs = (unsigned)(b.batch * b.beams) * (unsigned)a.parts;
  ProfScope ps(KID_BEAM, s);
  if (dtype == LAVA_BF16)
    hipLaunchKernelGGL(beam_rows_kernel<LAVA_BF16>, dim3(wgs), dim3(kBeamThreads), 0, s, a);
  else
    hipLaunchKernelGGL(beam_rows_kernel<LAVA_F32>, dim3(wgs), dim3(kBeamThreads), 0, s, a);
  const int32_t st = launch_status();
  if (st != LAVA_OK) return st;
  hipLaunchKernelGGL(beam_pick_kernel, dim3((unsigned)b.batch), dim3(kBeamThreads), 0, s, a);
  return launch_status();
}

}  // namespace lava
