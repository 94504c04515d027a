// What the decode steps over the packed cache and over pages share: the shape of a workgroup and its tile ring, lane moves (which
// the block tables' sums use too), and the tag by which a call knows its own flags.
#pragma once

#include <unistd.h>

#include <atomic>
#include <chrono>

#include "common.h"
#include "tile_ring.h"

namespace lava {

// A number that no other call of this process uses and that memory holds by chance once in 2^64 words: a mixed
// counter (a bijection of 64 bits) from a start of its own in every process.  The mixing and the counter's step are
// those of SplitMix64 (Steele, Lea, Flood, "Fast splittable pseudorandom number generators", 2014).
inline unsigned long long mix64(unsigned long long x) {
  x = (x ^ (x >> 30)) * 0xbf58476d1ce4e5b9ull;
  x = (x ^ (x >> 27)) * 0x94d049bb133111ebull;
  return x ^ (x >> 31);
}
inline unsigned long long next_tag() {
  static std::atomic<unsigned long long> next{
      mix64((unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() ^
            ((unsigned long long)getpid() << 40) ^ (unsigned long long)reinterpret_cast<uintptr_t>(&next))};
  for (;;) {
    const unsigned long long tag = mix64(next.fetch_add(0x9e3779b97f4a7c15ull, std::memory_order_relaxed));
    if (tag != 0ull) return tag;                            // 0 is "not published"
  }
}

namespace {

constexpr int kDecWaves = 4;
constexpr int kDecThreads = kDecWaves * 64;

// Two ring stages per wavefront (the K and the V tile of the moment): a workgroup then takes
// well under half of a compute unit's LDS, so two workgroups share a unit and the set-up of one
// overlaps the streaming of the other.
template <int DT, int D>
struct DecShape {
  using T = Tile<DT, D>;
  static constexpr int kStages = 2;
  static constexpr int kBpl = T::kRowBytes / 64;              // bytes of a row one lane owns
  static constexpr int kDpl = kBpl / Elem<DT>::kBytes;        // elements of a row one lane owns
  static_assert(kDpl == 1 || kDpl == 2, "one or two output columns per lane");
  static_assert(kDecWaves * kStages * T::kTileBytes >= kDecWaves * 8 * D * 4, "the ring doubles as the merge buffer");
};

template <int BYTES> struct RawBits;
template <> struct RawBits<2> { using type = unsigned short; };
template <> struct RawBits<4> { using type = unsigned int; };
template <> struct RawBits<8> { using type = uint2; };

// The kDpl elements of a row this lane owns, from their raw bits to floats.
template <int DT, int D>
__device__ __forceinline__ void unpack_v(const typename RawBits<DecShape<DT, D>::kBpl>::type& raw,
                                         float (&x)[DecShape<DT, D>::kDpl]) {
  using S = DecShape<DT, D>;
  if constexpr (DT == LAVA_BF16 && S::kDpl == 1) {
    x[0] = __uint_as_float((unsigned int)raw << 16);
  } else if constexpr (DT == LAVA_BF16) {
    x[0] = __uint_as_float(raw << 16);
    x[1] = __uint_as_float(raw & 0xffff0000u);
  } else if constexpr (S::kDpl == 1) {
    x[0] = __uint_as_float(raw);
  } else {
    x[0] = __uint_as_float(raw.x);
    x[1] = __uint_as_float(raw.y);
  }
}

// Values of a lane both kernels agree on, as scalars (no trip through the LDS unit).
__device__ __forceinline__ unsigned int lane_value(unsigned int x, int lane) {
  return (unsigned int)__builtin_amdgcn_readlane((int)x, lane);
}
__device__ __forceinline__ long long lane_value64(long long x, int lane) {
  const unsigned long long u = (unsigned long long)x;
  return (long long)(((unsigned long long)lane_value((unsigned int)(u >> 32), lane) << 32) | lane_value((unsigned int)u, lane));
}

template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned int dpp_add(unsigned int x) {
  return x + (unsigned int)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}

// Inclusive sum over the lanes.
__device__ __forceinline__ unsigned int wave_incl(unsigned int x) {
  x = dpp_add<0x111, 0xf>(x);
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);
  x = dpp_add<0x143, 0xc>(x);
  return x;
}

int padded_group(int G) { return G <= 1 ? 1 : G <= 2 ? 2 : G <= 4 ? 4 : 8; }

int device_cus() {
  static int cus = 0;
  if (cus == 0) {
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) == hipSuccess &&
        hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && n > 0)
      cus = n;
    else
      return 256;
  }
  return cus;
}

}  // namespace

}  // namespace lava
