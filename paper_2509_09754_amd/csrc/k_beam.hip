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
// Exponentials: e^x = 2^n e^f, n = rint(x log2 e), |f| <= ln 2 / 2, e^f by the polynomial of degree 7 whose largest relative error, 4.1e-11,
// is the least (coefficients by Remez's exchange).  15 64-bit instructions a token, at the rate of 32-bit ones on this
// device (2.4 ns a wavefront); with the polynomial of Taylor's series to degree 10, its exponent by ldexp and bounds from 64 readlanes a
// wavefront 64 groups of 8 beams over 131072 tokens took 85 us, now 61: rows 57 (107 MB of bf16 logits, 1.9 TB/s), pick 7.  Bound by the issue of
// instructions: more wavefronts (64 registers) or the chains of two or four tokens side by side take as long or longer.  One group of 4
// beams over 32000 tokens: 11.4 us, two launches of dependent look-ups.
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

// e^x for -700 <= x <= 0 (x below that: 10^-304, nothing beside the largest term, 1).  n log2 e + 1.5 * 2^52 has n in its last bits.
constexpr double kLog2e64 = 1.4426950408889634074, kLn2_64 = 0.69314718055994530942, kRound = 6755399441055744.0;
__device__ __forceinline__ double exp_of(double x) {
  x = fmax(x, -700.0);                                         // (NaN gives a number: whoever calls it looks for NaN by himself)
  const double t = fma(x, kLog2e64, kRound), n = t - kRound, f = fma(n, -kLn2_64, x);
  double p = 1.9775171620129632e-4;
  p = fma(p, f, 1.394818332942066e-3);
  p = fma(p, f, 8.3335610901591351e-3);
  p = fma(p, f, 4.1666225425460175e-2);
  p = fma(p, f, 1.6666665126137725e-1);
  p = fma(p, f, 5.0000001045362352e-1);
  p = fma(p, f, 1.0000000002430967);
  p = fma(p, f, 9.9999999996168187e-1);
  unsigned int hi = (unsigned int)(__double_as_longlong(p) >> 32);   // n to the exponent: one instruction, which the compiler makes five of
  asm("v_lshl_add_u32 %0, %1, 20, %0" : "+v"(hi) : "v"((unsigned int)__double_as_longlong(t)));
  return __hiloint2double((int)hi, (int)__double_as_longlong(p));
}

struct alignas(2) Bf16x8 { unsigned short x[8]; };
struct alignas(4) F32x4 { float x[4]; };

// Is beam `row` one whose logits count?
__device__ __forceinline__ bool is_live(const BeamArgs& b, int row) {
  return isfinite(b.scores[row]) && (b.done == nullptr || b.done[row] == 0);
}

// A bound that at least `count` of the lanes' values reach: the bits from LAST on of the count-th largest.
template <int LAST>
__device__ __forceinline__ unsigned int bound_of_wave(unsigned int x, int count) {
  unsigned int bound = 0u;
#pragma unroll
  for (int bit = 31; bit >= LAST; --bit) {
    const unsigned int next = bound | (1u << bit);
    bound = __popcll(__ballot(x >= next)) >= count ? next : bound;
  }
  return bound;
}

__device__ __forceinline__ float max_over_wave(float x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) x = fmaxf(x, __shfl_xor(x, m));
  return x;
}

// A candidate's rank is counted by eight lanes, each over every eighth of the others.
constexpr int kRankLanes = 8;
__device__ __forceinline__ int sum_of_ranks(int x) {
#pragma unroll
  for (int m = 1; m < kRankLanes; m <<= 1) x += __shfl_xor(x, m);
  return x;
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
  __shared__ float s_top[kBeamWaves];
  __shared__ unsigned int s_bound[kBeamWaves], s_bad[kBeamWaves];
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
  const unsigned int bound = bound_of_wave<DT == LAVA_BF16 ? 16 : 0>(most == -INFINITY ? 0u : score_key(most), b.n_out);
  const float of_wave = max_over_wave(most);
  const bool any_bad = __ballot(bad) != 0ull;
  if (lane == 0) {
    s_top[wave] = of_wave;
    s_bound[wave] = bound;
    s_bad[wave] = any_bad ? 1u : 0u;
  }
  if (threadIdx.x == 0) s_count = 0;
  __syncthreads();
  unsigned int limit_key = s_bound[0], wrong = s_bad[0];
  float m = s_top[0];
#pragma unroll
  for (int w = 1; w < kBeamWaves; ++w) {
    limit_key = s_bound[w] > limit_key ? s_bound[w] : limit_key;
    m = fmaxf(m, s_top[w]);
    wrong |= s_bad[w];
  }
  const long long out = (long long)row * a.parts + part;
  if (wrong != 0u || m == -INFINITY) {                         // uniform
    if (threadIdx.x == 0) {
      a.sum[out] = wrong != 0u ? NAN : 0.0;
      a.top[out] = -INFINITY;
    }
    if ((int)threadIdx.x < b.n_out) a.best[out * b.n_out + threadIdx.x] = 0ull;
    return;
  }
  // the bound as a logit; one that is no number's key, as all below -inf's: every token that can follow
  const float lowest = -3.402823466e38f;
  const float limit = limit_key < score_key(lowest) ? lowest : key_logit((unsigned long long)limit_key << 32);
  const double most64 = (double)m;                             // the difference first: m log2 e may be too large for its last bits to count
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) sum += exp_of((double)x[i] - most64);
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) sum += __shfl_xor(sum, s);
  if (lane == 0) s_sum[wave] = sum;
  // the list
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const bool in = x[i] >= limit;
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
    for (int i0 = 0; i0 < count; i0 += kBeamThreads / kRankLanes) {
      const int i = i0 + (int)threadIdx.x / kRankLanes;
      const unsigned long long key = s_list[i < count ? i : 0];
      int rank = 0;
      for (int j = threadIdx.x % kRankLanes; j < count; j += kRankLanes) rank += s_list[j] > key ? 1 : 0;
      rank = sum_of_ranks(rank);
      if (i < count && threadIdx.x % kRankLanes == 0 && rank < b.n_out) best[rank] = key;
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
constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64;
constexpr int kHeld = 4;                                       // candidates that a thread keeps
__global__ void __launch_bounds__(kPickThreads) beam_pick_kernel(const BeamKernelArgs a) {
  __shared__ Candidate s_list[kListed];
  __shared__ double s_base[kMostBeams];                        // log sum exp; NaN: no continuation
  __shared__ float s_score[kMostBeams];                        // read once: scores_out may be the same buffer
  __shared__ Candidate s_best[kPickWaves];
  __shared__ unsigned int s_bound[kPickWaves];
  __shared__ int s_over[kMostBeams], s_count;
  const BeamArgs& b = a.b;
  const int group = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // the first candidates' keys are on their way while the sums are formed
  const int each = a.parts * b.n_out, all = b.beams * each;
  const double inv_each = 1.0 / (double)each;                  // i / each: half a candidate off the border, so the product is exact enough
  auto beam_of = [&](int i) { return (int)(((double)i + 0.5) * inv_each); };
  unsigned long long key[kHeld];
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    const int i = threadIdx.x + u * kPickThreads;
    key[u] = i < all ? a.best[(long long)group * all + i] : 0ull;   // of a beam without continuations whatever is there: not used
  }
  for (int i = wave; i < b.beams; i += kPickWaves) {
    const int row = group * b.beams + i;
    const float score = b.scores[row];
    const bool over = b.done != nullptr && b.done[row] != 0;
    double base = NAN;
    if (isfinite(score) && !over) {                            // uniform
      float m = -INFINITY;
      for (int q = lane; q < a.parts; q += 64) m = fmaxf(m, a.top[(long long)row * a.parts + q]);
      m = max_over_wave(m);
      double sum = 0.0;
      for (int q = lane; q < a.parts; q += 64) {
        const float t = a.top[(long long)row * a.parts + q];
        const double z = a.sum[(long long)row * a.parts + q];
        sum += isnan(z) ? z : t == -INFINITY ? 0.0 : z * exp_of((double)t - (double)m);
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
  auto candidate = [&](int i, unsigned long long of) {
    Candidate r = {0ull, 0ull, beam_of(i)};
    const double base = s_base[r.beam], score = (double)s_score[r.beam];
    if (isnan(base)) return r;
    if (s_over[r.beam] != 0) {
      if (i != r.beam * each) return r;
      r.c = order_of(score);
      r.key = token_key(0.0f, (unsigned int)b.pad_token);
      return r;
    }
    r.key = of;
    if (of != 0ull) r.c = order_of(score + ((double)key_logit(of) - base));
    return r;
  };
  auto stored = [&](int i) { return !isnan(s_base[beam_of(i)]) && s_over[beam_of(i)] == 0 ? a.best[(long long)group * all + i] : 0ull; };
  Candidate mine[kHeld];
  unsigned int top = 0u;
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    const int i = threadIdx.x + u * kPickThreads;
    mine[u] = Candidate{0ull, 0ull, 0};
    if (i < all) mine[u] = candidate(i, key[u]);
    top = (unsigned int)(mine[u].c >> 32) > top ? (unsigned int)(mine[u].c >> 32) : top;
  }
  for (int i = threadIdx.x + kHeld * kPickThreads; i < all; i += kPickThreads) {
    const unsigned int y = (unsigned int)(candidate(i, stored(i)).c >> 32);
    top = y > top ? y : top;
  }
  const unsigned int bound = bound_of_wave<0>(top, b.n_out);
  if (lane == 0) s_bound[wave] = bound;
  __syncthreads();
  unsigned int limit = s_bound[0];
#pragma unroll
  for (int w = 1; w < kPickWaves; ++w) limit = s_bound[w] > limit ? s_bound[w] : limit;
  auto list = [&](const Candidate& r) {
    if (r.c == 0ull || (unsigned int)(r.c >> 32) < limit) return;
    const int at = atomicAdd(&s_count, 1);
    if (at < kListed) s_list[at] = r;
  };
#pragma unroll
  for (int u = 0; u < kHeld; ++u) list(mine[u]);
  for (int i = threadIdx.x + kHeld * kPickThreads; i < all; i += kPickThreads) list(candidate(i, stored(i)));
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
    for (int i0 = 0; i0 < count; i0 += kPickThreads / kRankLanes) {
      const int i = i0 + (int)threadIdx.x / kRankLanes;
      const Candidate r = s_list[i < count ? i : 0];
      int rank = 0;
      for (int j = threadIdx.x % kRankLanes; j < count; j += kRankLanes) rank += before(s_list[j], r) ? 1 : 0;
      rank = sum_of_ranks(rank);
      if (i < count && threadIdx.x % kRankLanes == 0 && rank < b.n_out) write(rank, r);
    }
    for (int i = count + (int)threadIdx.x; i < b.n_out; i += kPickThreads) write(i, Candidate{0ull, 0ull, 0});
    return;
  }
  Candidate last = {~0ull, ~0ull, -1};
  for (int k = 0; k < b.n_out; ++k) {
    Candidate r = {0ull, 0ull, 0};
    for (int i = threadIdx.x; i < all; i += kPickThreads) {
      const Candidate y = candidate(i, stored(i));
      if (y.c != 0ull && before(last, y) && before(y, r)) r = y;
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const Candidate y = {__shfl_xor(r.c, s), __shfl_xor(r.key, s), __shfl_xor(r.beam, s)};
      if (before(y, r)) r = y;
    }
    if (lane == 0) s_best[wave] = r;
    __syncthreads();
    for (int w = 0; w < kPickWaves; ++w)
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
  hipLaunchKernelGGL(beam_pick_kernel, dim3((unsigned)b.batch), dim3(kPickThreads), 0, s, a);
  return launch_status();
}

}  // namespace lava
