// Pages of the paged cache: block tables and slot maps of a step, and the gather of an eviction's
// survivors into pages.
//
// A step's tables are exclusive sums over the heads in order: head i needs ceil((old + add) / P) - ceil(old / P)
// pages and pops them behind those of the heads before it.  Everything else follows from the sums: which page a
// new block gets is one look-up in the stack, which slot a new row has is one look-up in the stack or the table.
//
// A step with little to write, as a decode step is, is one launch of one workgroup: a chain of four trips to memory (64 sequences on
// 8 heads 6.0 us with the host's share).  For a large one a first launch forms the sums, a workgroup for every 1024 heads, and every
// workgroup of the second adds up the workgroups' totals for itself; that launch fills the device and is bound by the slots it
// writes, 8 bytes a row (559 thousand tokens on 8 heads, 36 MB of slots: 17.1 us both launches, 8.3 at a copy's rate; a fifth
// of it is the first launch, the rest four dependent trips to memory around the writes).  Sequences that leave cost a launch
// between the two, which puts their pages on the stack before any is taken (16384 heads, a quarter leaving: 18.5 us).
#include "common.h"
#include "decode_parts.h"

namespace lava {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;

// What the sums' launch leaves in the workspace.  Heads, and sequences, are summed in chunks, at most kMaxChunks of them.
constexpr int kMaxChunks = 256;
struct ChunkTotals {
  unsigned long long need, back;   // of a chunk of heads: pages needed, pages given back; of sequences: tokens, -
  int error;                       // LAVA_PAGES_* bits
  int n_free;                      // of the first chunk of heads: the stack's pages when the step began (n_free_out may be n_free)
};
struct PlanLayout {
  size_t off_old;        // int [heads]   rows every head starts the step with (0 where it is over)
  size_t off_need;       // int [heads]   pages needed by the heads of the chunk before
  size_t off_back;       // int [heads]   pages given back by them
  size_t off_tok;        // int [batch]   new tokens of the sequences of the chunk before
  size_t off_pos;        // int [batch]   position of every sequence's first new token
  size_t bytes;          // at 0: ChunkTotals [2][kMaxChunks], of the heads' chunks and of the sequences'
};
__host__ __device__ inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
__host__ __device__ inline PlanLayout plan_layout(int batch, int heads) {
  PlanLayout l;
  l.off_old = up256(2 * kMaxChunks * sizeof(ChunkTotals));
  l.off_need = l.off_old + up256((size_t)heads * 4);
  l.off_back = l.off_need + up256((size_t)heads * 4);
  l.off_tok = l.off_back + up256((size_t)heads * 4);
  l.off_pos = l.off_tok + up256((size_t)batch * 4);
  l.bytes = l.off_pos + up256((size_t)batch * 4);
  return l;
}

// Sum over the lanes of values below 2^48, in two halves of 24 bits and more.
__device__ __forceinline__ unsigned long long wave_total(unsigned long long x) {
  const unsigned int lo = lane_value(wave_incl((unsigned int)x & 0xffffffu), 63), hi = lane_value(wave_incl((unsigned int)(x >> 24)), 63);
  return ((unsigned long long)hi << 24) + lo;
}

// Exclusive sums of a workgroup's values x[u] of items u * kPlanThreads + thread, in the order of the items.  32 bits: where they
// could overflow the 64-bit totals refuse the step.
template <int PER>
__device__ __forceinline__ void plan_scan(unsigned int (&x)[PER], unsigned int* s_part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  unsigned int incl[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    incl[u] = wave_incl(x[u]);
    if (lane == 63) s_part[u * kPlanWaves + wave] = incl[u];
  }
  __syncthreads();
  if (wave == 0) {                                                 // sums of the wavefronts' sums, 64 at a time
    unsigned int carry = 0u;
    for (int i0 = 0; i0 < PER * kPlanWaves; i0 += 64) {
      const int i = i0 + lane;
      const unsigned int v = i < PER * kPlanWaves ? s_part[i] : 0u, s = wave_incl(v);
      if (i < PER * kPlanWaves) s_part[i] = carry + s - v;
      carry += lane_value(s, 63);
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < PER; ++u) x[u] = s_part[u * kPlanWaves + wave] + incl[u] - x[u];
  __syncthreads();
}

struct HeadStep {
  int old, add, need, back, error;
};

// What head hb does in this step.
__device__ __forceinline__ HeadStep head_step(const PageTablesArgs& a, int hb) {
  const int b = hb / a.heads;
  const bool over = a.release != nullptr && a.release[b] != 0;
  const int rows = a.st.head_rows[hb];
  const int add = a.head_counts != nullptr ? a.head_counts[hb] : a.n_new != nullptr ? a.n_new[b] : 0;
  HeadStep h;
  h.error = 0;
  const long long most = (long long)a.max_blocks << a.page_shift;
  const int mask = (1 << a.page_shift) - 1;
  if (rows < 0 || rows > most || add < 0) h.error = LAVA_PAGES_INVALID;
  h.back = over && h.error == 0 ? (int)(((long long)rows + mask) >> a.page_shift) : 0;
  h.old = over || h.error != 0 ? 0 : rows;
  h.add = h.error != 0 ? 0 : add;
  if ((long long)h.old + h.add > most) {
    h.error |= LAVA_PAGES_BLOCKS;
    h.add = 0;
  }
  h.need = (int)(((long long)h.old + h.add + mask) >> a.page_shift) - (int)(((long long)h.old + mask) >> a.page_shift);
  return h;
}

// The sums as the steps that use them see them: in LDS from the one workgroup (chunk = 31: one chunk of all), or in the workspace with
// the sums of the chunks before in LDS.
struct PlanSums {
  const int *old, *need, *back, *tok, *pos;
  const int *base_need, *base_back, *base_tok;   // [chunks]
  int chunk;                                       // log2 of a chunk
  int heads, batch, total_need, total_back, total_tok;
  __device__ __forceinline__ int need_at(int hb) const { return hb < heads ? need[hb] + base_need[hb >> chunk] : total_need; }
  __device__ __forceinline__ int back_at(int hb) const { return hb < heads ? back[hb] + base_back[hb >> chunk] : total_back; }
  __device__ __forceinline__ int tok_at(int b) const { return b < batch ? tok[b] + base_tok[b >> chunk] : total_tok; }
};

// Pages of the sequences that are over, onto the stack: a wavefront per head.
__device__ __forceinline__ void give_back(const PageTablesArgs& a, const PlanSums& w, int free_pages, int first, int step) {
  const int lane = threadIdx.x & 63, heads = a.batch * a.heads;
  for (int hb = first; hb < heads; hb += step) {
    const int at = w.back_at(hb), n = w.back_at(hb + 1) - at;
    const int* table = a.st.block_table + (long long)hb * a.max_blocks;
    for (int j = lane; j < n; j += 64) a.st.free_pages[free_pages + at + j] = table[j];
  }
}

// Tables and counts of the heads, LANES threads a head: one where heads take a page now and then, more where they may take many.
template <int LANES>
__device__ __forceinline__ void fill_heads(const PageTablesArgs& a, const PlanSums& w, int top, int first, int step) {
  constexpr int kBatch = LANES > 1 ? 4 : 1;                            // look-ups a thread has in flight
  const int lane = (int)threadIdx.x % LANES, heads = a.batch * a.heads, mask = (1 << a.page_shift) - 1;
  for (int hb = first; hb < heads; hb += step) {
    const int old = w.old[hb], start = w.need_at(hb), need = w.need_at(hb + 1) - start;
    int* table = a.st.block_table + (long long)hb * a.max_blocks + ((old + mask) >> a.page_shift);
    const int* fresh = a.st.free_pages + (top - 1 - start);
    for (int j0 = lane; j0 < need; j0 += LANES * kBatch) {
      int page[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) page[i] = j0 + LANES * i < need ? fresh[-(j0 + LANES * i)] : 0;
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (j0 + LANES * i < need) table[j0 + LANES * i] = page[i];
    }
    if (lane == 0) {
      const int add = a.head_counts != nullptr ? a.head_counts[hb] : a.n_new != nullptr ? a.n_new[hb / a.heads] : 0;
      a.st.head_rows_out[hb] = old + add;
    }
  }
}

// Slots and positions of `count` (token, head) places from place e on, `stride` apart; `tokens` of the tokens are real.
__device__ __forceinline__ void fill_slots(const PageTablesArgs& a, const PlanSums& w, int top, int tokens, unsigned int e,
                                           unsigned int stride, int count) {
  const unsigned int all = (unsigned int)(a.max_tokens * a.heads), heads = (unsigned int)a.heads;
  const int mask = (1 << a.page_shift) - 1;
  const bool same_head = stride % heads == 0u;                       // uniform
  unsigned int t = e / heads, g = e - t * heads;
  int b = -1, end = 0, begin = 0, old = 0, start = 0, pos = 0, hb = 0;   // of the sequence (b >= 0) and its head
  for (int i = 0; i < count && e < all; ++i, e += stride) {
    if (i > 0) {
      if (same_head) {
        t += stride / heads;
      } else {
        t = e / heads;
        g = e - t * heads;
      }
    }
    if ((int)t >= tokens) {
      if (a.slots != nullptr) a.slots[e] = -1;
      if (a.positions != nullptr && g == 0u) a.positions[t] = -1;
      continue;
    }
    if (b < 0 || (int)t >= end || !same_head) {
      int lo = b < 0 ? 0 : b, hi = a.batch - 1;                       // the last sequence that starts at or before t
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (w.tok_at(mid) <= (int)t) lo = mid; else hi = mid - 1;
      }
      b = lo;
      begin = w.tok_at(b);
      end = w.tok_at(b + 1);
      hb = b * a.heads + (int)g;
      old = w.old[hb];
      start = w.need_at(hb);
      pos = w.pos[b];
    }
    if (a.positions != nullptr && g == 0u) a.positions[t] = pos + (int)t - begin;
    if (a.slots == nullptr) continue;
    const int r = old + (int)t - begin, block = r >> a.page_shift, owned = (old + mask) >> a.page_shift;
    const int page = block < owned ? a.st.block_table[(long long)hb * a.max_blocks + block]
                                   : a.st.free_pages[top - 1 - start - (block - owned)];
    a.slots[e] = ((long long)page << a.page_shift) + (r & mask);
  }
}

// The same for the 256 * ITEMS places from place e0 on, by a workgroup of 256 threads.  Where all of them are tokens of one sequence, as
// most of a prompt's are, a thread stays with its head and its look-ups are independent of each other; that takes a head count that
// divides 256 (16 prompts on 8 heads 17 us both launches, on 10 and 12 heads, place by place, 31 and 32.5).
template <int ITEMS>
__device__ __forceinline__ void fill_slots_wide(const PageTablesArgs& a, const PlanSums& w, int top, int tokens, unsigned int e0) {
  const unsigned int all = (unsigned int)(a.max_tokens * a.heads), heads = (unsigned int)a.heads;
  if (256u % heads == 0u && a.slots != nullptr && e0 + 256u * ITEMS <= all) {
    const int t_first = (int)(e0 / heads), t_last = (int)((e0 + 256u * ITEMS - 1u) / heads);
    if (t_last < tokens) {
      int lo = 0, hi = a.batch - 1;                                  // uniform: the last sequence that starts at or before t_first
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (__builtin_amdgcn_readfirstlane(w.tok_at(mid)) <= t_first) lo = mid; else hi = mid - 1;
      }
      const int begin = w.tok_at(lo);
      if (t_last < w.tok_at(lo + 1)) {
        const unsigned int e = e0 + threadIdx.x, t = e / heads, g = e - t * heads;
        const int mask = (1 << a.page_shift) - 1, hb = lo * a.heads + (int)g, step = (int)(256u / heads);
        const int old = w.old[hb], owned = (old + mask) >> a.page_shift, i0 = (int)t - begin;
        const int* table = a.st.block_table + (long long)hb * a.max_blocks;
        const int* fresh = a.st.free_pages + (top - 1 - w.need_at(hb) + owned);   // the page of new block j is fresh[-j]
        int page[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
          const int block = (old + i0 + i * step) >> a.page_shift;
          page[i] = *(block < owned ? table + block : fresh - block);
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
          const int r = old + i0 + i * step;
          a.slots[e + 256u * i] = ((long long)page[i] << a.page_shift) + (r & mask);
        }
        if (a.positions != nullptr && g == 0u) {
          const int pos = w.pos[lo] + i0;
          for (int i = 0; i < ITEMS; ++i) a.positions[t + (unsigned int)(i * step)] = pos + i * step;
        }
        return;
      }
    }
  }
  fill_slots(a, w, top, tokens, e0 + threadIdx.x, 256u, ITEMS);
}

// What sequence b does: its tokens (0 where it cannot be), its first position.
__device__ __forceinline__ int seq_step(const PageTablesArgs& a, int b, int& pos, int& error) {
  const int n = a.n_new != nullptr ? a.n_new[b] : 0;
  pos = a.release != nullptr && a.release[b] != 0 ? 0 : a.st.seq_pos[b];
  if (n >= 0 && pos >= 0 && (long long)pos + n < (long long)1 << 31) return n;
  error |= LAVA_PAGES_INVALID;
  return 0;
}

// May the step be carried out?
__device__ __forceinline__ int verdict(const PageTablesArgs& a, int error, long long free_pages, unsigned long long need,
                                       unsigned long long back, unsigned long long tokens) {
  if (free_pages < 0 || free_pages + (long long)back > a.n_pages) error |= LAVA_PAGES_INVALID;
  else if ((long long)need > free_pages + (long long)back) error |= LAVA_PAGES_EXHAUSTED;
  if (a.max_tokens > 0 && tokens > (unsigned long long)a.max_tokens) error |= LAVA_PAGES_TOKENS;
  return error;
}

// A whole step by one workgroup.
constexpr int kOnePer = 2, kOneHeads = kOnePer * kPlanThreads;
__global__ void __launch_bounds__(kPlanThreads) page_step_kernel(const PageTablesArgs a) {
  __shared__ unsigned int s_part[kOnePer * kPlanWaves];
  __shared__ unsigned long long s_total[3];                          // pages needed, pages given back, tokens
  __shared__ int s_error, s_zero;
  __shared__ int s_old[kOneHeads], s_need[kOneHeads], s_back[kOneHeads], s_tok[kOneHeads], s_pos[kOneHeads];
  const int heads = a.batch * a.heads;
  if (threadIdx.x == 0) s_error = s_zero = 0;
  if (threadIdx.x < 3) s_total[threadIdx.x] = 0ull;
  int error = 0;
  unsigned int need[kOnePer], back[kOnePer], tok[kOnePer];
  unsigned long long all_need = 0ull, all_back = 0ull, all_tok = 0ull;
#pragma unroll
  for (int u = 0; u < kOnePer; ++u) {
    const int hb = u * kPlanThreads + (int)threadIdx.x;
    HeadStep h = {0, 0, 0, 0, 0};
    if (hb < heads) {
      h = head_step(a, hb);
      s_old[hb] = h.old;
    }
    int n = 0, pos = 0;
    if (hb < a.batch) {
      n = seq_step(a, hb, pos, error);
      s_pos[hb] = pos;
    }
    error |= h.error;
    all_need += need[u] = (unsigned int)h.need;
    all_back += back[u] = (unsigned int)h.back;
    all_tok += tok[u] = (unsigned int)n;
  }
  __syncthreads();                                                   // the totals are zero
  all_need = wave_total(all_need);
  all_tok = wave_total(all_tok);
  if (a.release != nullptr) all_back = wave_total(all_back);         // uniform
  if ((threadIdx.x & 63) == 0) {
    if (all_need != 0ull) atomicAdd(&s_total[0], all_need);
    if (a.release != nullptr && all_back != 0ull) atomicAdd(&s_total[1], all_back);
    if (all_tok != 0ull) atomicAdd(&s_total[2], all_tok);
  }
  if (error != 0) atomicOr(&s_error, error);
  plan_scan<kOnePer>(need, s_part);
  if (a.release != nullptr) plan_scan<kOnePer>(back, s_part);
  if (a.max_tokens > 0) plan_scan<kOnePer>(tok, s_part);
#pragma unroll
  for (int u = 0; u < kOnePer; ++u) {
    const int hb = u * kPlanThreads + (int)threadIdx.x;
    s_need[hb] = (int)need[u];
    s_back[hb] = (int)back[u];
    s_tok[hb] = (int)tok[u];
  }
  const long long free_pages = a.st.n_free[0];
  __syncthreads();                                                   // every thread has read n_free, which n_free_out may be
  error = verdict(a, s_error, free_pages, s_total[0], s_total[1], s_total[2]);   // the same in every thread
  const int top = (int)(free_pages + (long long)s_total[1]);
  if (threadIdx.x == 0 && error != 0 && a.st.error != nullptr) atomicOr(a.st.error, error);
  const PlanSums w = {s_old, s_need, s_back, s_tok, s_pos, &s_zero, &s_zero, &s_zero, 31, heads, a.batch, (int)s_total[0], (int)s_total[1], (int)s_total[2]};
  const int wave = threadIdx.x >> 6;
  if (error == 0 && a.release != nullptr) {
    give_back(a, w, (int)free_pages, wave, kPlanWaves);
    __syncthreads();                                                 // the stack's new pages, for this workgroup to read
  }
  if (a.max_tokens > 0) {
    const unsigned int places = (unsigned int)(a.max_tokens * a.heads);
    fill_slots(a, w, top, error != 0 ? 0 : w.total_tok, threadIdx.x, kPlanThreads, (int)((places + kPlanThreads - 1) / kPlanThreads));
  }
  if (error == 0) {
    fill_heads<1>(a, w, top, threadIdx.x, kPlanThreads);
  } else {
    for (int hb = threadIdx.x; hb < heads; hb += kPlanThreads) a.st.head_rows_out[hb] = a.st.head_rows[hb];
  }
  for (int b = threadIdx.x; b < a.batch; b += kPlanThreads)
    a.st.seq_pos_out[b] = error != 0 ? a.st.seq_pos[b] : s_pos[b] + (a.n_new != nullptr ? a.n_new[b] : 0);
  if (threadIdx.x == 0) a.st.n_free_out[0] = error != 0 ? (int)free_pages : top - w.total_need;
}

// Sums of the chunks: the first `head_chunks` workgroups of heads, the others of sequences, PER * 1024 each.
template <int PER>
__global__ void __launch_bounds__(kPlanThreads) page_sums_kernel(const PageTablesArgs a, const int head_chunks) {
  __shared__ unsigned int s_part[PER * kPlanWaves];
  __shared__ unsigned long long s_total[2];
  __shared__ int s_error;
  const bool of_heads = (int)blockIdx.x < head_chunks;
  const int chunk = of_heads ? blockIdx.x : blockIdx.x - head_chunks, items = of_heads ? a.batch * a.heads : a.batch;
  const PlanLayout l = plan_layout(a.batch, a.batch * a.heads);
  char* ws = static_cast<char*>(a.ws);
  if (threadIdx.x == 0) s_error = 0;
  if (threadIdx.x < 2) s_total[threadIdx.x] = 0ull;
  int error = 0;
  unsigned int x[PER], y[PER];
  unsigned long long all_x = 0ull, all_y = 0ull;
  int* first = reinterpret_cast<int*>(ws + (of_heads ? l.off_old : l.off_pos));
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = (chunk * PER + u) * kPlanThreads + (int)threadIdx.x;
    x[u] = y[u] = 0u;
    if (i < items) {
      if (of_heads) {
        const HeadStep h = head_step(a, i);
        error |= h.error;
        x[u] = (unsigned int)h.need;
        y[u] = (unsigned int)h.back;
        first[i] = h.old;
      } else {
        int pos;
        x[u] = (unsigned int)seq_step(a, i, pos, error);
        first[i] = pos;
      }
    }
    all_x += x[u];
    all_y += y[u];
  }
  __syncthreads();
  const bool backs = of_heads && a.release != nullptr;               // uniform
  all_x = wave_total(all_x);
  if (backs) all_y = wave_total(all_y);
  if ((threadIdx.x & 63) == 0) {
    atomicAdd(&s_total[0], all_x);
    if (backs) atomicAdd(&s_total[1], all_y);
  }
  if (error != 0) atomicOr(&s_error, error);
  plan_scan<PER>(x, s_part);
  if (backs) plan_scan<PER>(y, s_part);
  int* out = reinterpret_cast<int*>(ws + (of_heads ? l.off_need : l.off_tok));
  int* out_back = reinterpret_cast<int*>(ws + l.off_back);
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = (chunk * PER + u) * kPlanThreads + (int)threadIdx.x;
    if (i < items) {
      out[i] = (int)x[u];
      if (backs) out_back[i] = (int)y[u];
    }
  }
  if (threadIdx.x == 0)
    reinterpret_cast<ChunkTotals*>(ws)[(of_heads ? 0 : kMaxChunks) + chunk] = ChunkTotals{s_total[0], s_total[1], s_error, a.st.n_free[0]};
}

// What a workgroup of 256 threads of the second launch needs of the totals: sums of the chunks before, and the verdict.
constexpr int kFewSequences = 1024;   // as many as one chunk holds: their tokens' sums are looked up in LDS
struct FillPlan {
  int base_need[kMaxChunks], base_back[kMaxChunks], base_tok[kMaxChunks];
  unsigned long long part[3][4];
  int error;
  int tok[kFewSequences];
};
__device__ __forceinline__ unsigned long long lane_sum64(unsigned long long x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned int lo = __shfl_up((unsigned int)x, d), hi = __shfl_up((unsigned int)(x >> 32), d);
    if (lane >= d) x += ((unsigned long long)hi << 32) | lo;
  }
  return x;
}
__device__ __forceinline__ PlanSums add_up(const PageTablesArgs& a, int chunk, FillPlan& f, bool with_tokens, int& error, int& top, int& n_free) {
  const char* ws = static_cast<const char*>(a.ws);
  const int heads = a.batch * a.heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int head_chunks = ((heads - 1) >> chunk) + 1, seq_chunks = ((a.batch - 1) >> chunk) + 1;
  const PlanLayout l = plan_layout(a.batch, heads);
  const ChunkTotals* totals = reinterpret_cast<const ChunkTotals*>(ws);
  const int* tok = reinterpret_cast<const int*>(ws + l.off_tok);
  if (with_tokens && a.batch <= kFewSequences) {                       // uniform
    for (int b = threadIdx.x; b < a.batch; b += 256) f.tok[b] = tok[b];
    tok = f.tok;
  }
  if (head_chunks == 1 && seq_chunks == 1) {                           // nothing to add up
    const ChunkTotals h = totals[0], s = totals[kMaxChunks];
    if (threadIdx.x == 0) f.base_need[0] = f.base_back[0] = f.base_tok[0] = 0;
    __syncthreads();
    n_free = h.n_free;
    error = verdict(a, h.error | s.error, n_free, h.need, h.back, s.need);
    top = (int)(n_free + (long long)h.back);
    return {reinterpret_cast<const int*>(ws + l.off_old),  reinterpret_cast<const int*>(ws + l.off_need),
            reinterpret_cast<const int*>(ws + l.off_back), tok,
            reinterpret_cast<const int*>(ws + l.off_pos),  f.base_need, f.base_back, f.base_tok, chunk, heads, a.batch,
            (int)h.need, (int)h.back, (int)s.need};
  }
  ChunkTotals h = {0ull, 0ull, 0, 0}, s = h;
  if ((int)threadIdx.x < head_chunks) h = totals[threadIdx.x];
  if ((int)threadIdx.x < seq_chunks) s = totals[kMaxChunks + threadIdx.x];
  if (threadIdx.x == 0) f.error = 0;
  unsigned long long x[3] = {h.need, h.back, s.need}, incl[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    incl[i] = lane_sum64(x[i]);
    if (lane == 63) f.part[i][wave] = incl[i];
  }
  __syncthreads();
  if ((h.error | s.error) != 0) atomicOr(&f.error, h.error | s.error);
  unsigned long long before[3] = {0ull, 0ull, 0ull}, total[3] = {0ull, 0ull, 0ull};
#pragma unroll
  for (int i = 0; i < 3; ++i)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      if (v < wave) before[i] += f.part[i][v];
      total[i] += f.part[i][v];
    }
  f.base_need[threadIdx.x] = (int)(before[0] + incl[0] - x[0]);
  f.base_back[threadIdx.x] = (int)(before[1] + incl[1] - x[1]);
  f.base_tok[threadIdx.x] = (int)(before[2] + incl[2] - x[2]);
  __syncthreads();
  n_free = totals[0].n_free;
  error = verdict(a, f.error, n_free, total[0], total[1], total[2]);
  top = (int)(n_free + (long long)total[1]);
  return {reinterpret_cast<const int*>(ws + l.off_old),  reinterpret_cast<const int*>(ws + l.off_need),
          reinterpret_cast<const int*>(ws + l.off_back), tok,
          reinterpret_cast<const int*>(ws + l.off_pos),  f.base_need, f.base_back, f.base_tok, chunk, heads, a.batch,
          (int)total[0], (int)total[1], (int)total[2]};
}

__global__ void __launch_bounds__(256) page_return_kernel(const PageTablesArgs a, const int chunk) {
  static_assert(kMaxChunks == 256, "a thread for every chunk");
  __shared__ FillPlan f;
  int error, top, n_free;
  const PlanSums w = add_up(a, chunk, f, false, error, top, n_free);
  if (error != 0) return;
  give_back(a, w, n_free, blockIdx.x * 4 + (threadIdx.x >> 6), gridDim.x * 4);
}

// The first `head_wgs` workgroups take the heads (one each, or one for each wavefront), the others the tokens.
constexpr int kSlotItems = 8;   // slots a thread writes: 4.5 million 4 19.9 us, 8 18.7, 16 20.6; 2.6 million one 21.4, 8 14.0; 0.6 million 10.4 with both
// One workgroup finishes a step of so few places (slots, and table entries that may change hands) sooner than two launches begin:
// 2560 slots 8.1 us (two launches 8.6), 3840 8.9 (8.6), 16000 15.4 (8.6); 512 heads that take a page now and then 6.8 (8.7).
// Where a table may fill by any number of pages it is the table that counts, whatever happens then: without maps 8 heads that take 4096
// pages each 479 us (two launches 7.4), 2048 heads that take 63 each 150 (7.5), 512 that take a page now and then 5.0 (7.2).
constexpr long long kOnePlaces = 2560;
template <int ITEMS>
__global__ void __launch_bounds__(256) page_fill_kernel(const PageTablesArgs a, const int chunk, const int head_wgs) {
  __shared__ FillPlan f;
  int error, top, n_free;
  const PlanSums w = add_up(a, chunk, f, (int)blockIdx.x >= head_wgs, error, top, n_free);
  if ((int)blockIdx.x >= head_wgs) {
    fill_slots_wide<ITEMS>(a, w, top, error != 0 ? 0 : w.total_tok, (blockIdx.x - head_wgs) * (256u * ITEMS));
    return;
  }
  const int heads = a.batch * a.heads;
  if (error == 0) {
    if (heads <= head_wgs) fill_heads<256>(a, w, top, blockIdx.x, head_wgs);
    else fill_heads<64>(a, w, top, blockIdx.x * 4 + (threadIdx.x >> 6), head_wgs * 4);
  } else {
    for (int hb = blockIdx.x * 256 + (int)threadIdx.x; hb < heads; hb += head_wgs * 256) a.st.head_rows_out[hb] = a.st.head_rows[hb];
  }
  for (int b = blockIdx.x * 256 + (int)threadIdx.x; b < a.batch; b += head_wgs * 256)
    a.st.seq_pos_out[b] = error != 0 ? a.st.seq_pos[b] : w.pos[b] + (a.n_new != nullptr ? a.n_new[b] : 0);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.st.n_free_out[0] = error != 0 ? n_free : top - w.total_need;
    if (error != 0 && a.st.error != nullptr) atomicOr(a.st.error, error);
  }
}

}  // namespace

size_t page_tables_bytes(int32_t batch, int32_t n_kv_heads) { return plan_layout(batch, batch * n_kv_heads).bytes; }

int32_t launch_page_tables(const PageTablesArgs& a, hipStream_t s) {
  const long long heads = (long long)a.batch * a.heads, places = a.max_tokens * a.heads;
  // Written by the one workgroup alone: every slot, a count per head and, where heads take or give back any number of pages, up
  // to the whole table.  Tokens with maps cannot take more than the maps have room for; without maps nothing else bounds them.
  const bool unbounded = a.head_counts != nullptr || a.release != nullptr || (a.n_new != nullptr && a.max_tokens == 0);
  const long long pages = unbounded ? heads * a.max_blocks : 0;
  const bool one = heads <= kOneHeads && places + pages <= kOnePlaces;
  if (one) {
    ProfScope ps(KID_PAGE_PLAN, s);
    hipLaunchKernelGGL(page_step_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
    return launch_status();
  }
  const int chunk = heads <= (long long)kMaxChunks * kPlanThreads ? 10 : 12;   // 1024 or 4096 heads a chunk
  const int head_chunks = (int)((heads - 1) >> chunk) + 1, seq_chunks = ((a.batch - 1) >> chunk) + 1;
  {
    ProfScope ps(KID_PAGE_PLAN, s);
    const dim3 grid((unsigned)(head_chunks + seq_chunks)), block(kPlanThreads);
    if (chunk == 10) hipLaunchKernelGGL(page_sums_kernel<1>, grid, block, 0, s, a, head_chunks);
    else hipLaunchKernelGGL(page_sums_kernel<4>, grid, block, 0, s, a, head_chunks);
  }
  int32_t st = launch_status();
  if (st != LAVA_OK) return st;
  // a workgroup a head; more than 1024 heads share as many, a wavefront a head
  const long long head_wgs = heads < 1024 ? heads : 1024;
  if (a.release != nullptr) {
    ProfScope ps(KID_PAGE_FILL, s);
    hipLaunchKernelGGL(page_return_kernel, dim3((unsigned)head_wgs), dim3(256), 0, s, a, chunk);
    st = launch_status();
    if (st != LAVA_OK) return st;
  }
  // one place a thread where that is at most 1024 workgroups, else kSlotItems
  const bool many = places > 256 * 1024;
  const long long per = 256 * (many ? kSlotItems : 1), slot_wgs = (places + per - 1) / per;
  const dim3 grid((unsigned)(head_wgs + slot_wgs)), block(256);
  ProfScope ps(KID_PAGE_FILL, s);
  if (many) hipLaunchKernelGGL(page_fill_kernel<kSlotItems>, grid, block, 0, s, a, chunk, (int)head_wgs);
  else hipLaunchKernelGGL(page_fill_kernel<1>, grid, block, 0, s, a, chunk, (int)head_wgs);
  return launch_status();
}

// ------------------------------------------------------------------------------------------
// The gather of an eviction's survivors into pages: bound by HBM, 4 * d_h * elem bytes a row.  A row is
// moved by (row bytes / 16) lanes; the workgroups of a problem walk over its survivors.  131072 rows of 2 x 256 bytes (16 prompts):
// 32.0 us, 4.2 TB/s read and written, of rows that lie apart on both sides; two, four and eight rows in flight a lane took 32.9,
// 34.7 and 38.0.
// ------------------------------------------------------------------------------------------
namespace {

constexpr int kGatherThreads = 256;
constexpr int kGatherMaxHeads = 64;

struct PagedBatch {
  char *k, *v;
  int32_t* pos;
  long long n_pages;
  int page_shift, max_blocks, n_heads;
  lava_paged_compact_problem p[kMaxSelProblems];
};

template <int LPR>
__global__ void __launch_bounds__(kGatherThreads) compact_paged_kernel(const PagedBatch a) {
  const lava_paged_compact_problem pr = a.p[blockIdx.y];
  constexpr int kRowsPerBlock = kGatherThreads / LPR;
  if ((long long)blockIdx.x * kRowsPerBlock >= pr.capacity) return;
  __shared__ long long s_off[kGatherMaxHeads + 1], s_src[kGatherMaxHeads + 1];
  __shared__ int s_first[kGatherMaxHeads];
  const int heads = a.n_heads;
  if ((int)threadIdx.x <= heads) {
    s_off[threadIdx.x] = (long long)pr.head_offsets[threadIdx.x];
    s_src[threadIdx.x] = pr.src_offsets ? (long long)pr.src_offsets[threadIdx.x] : (long long)threadIdx.x * pr.src_rows;
    if ((int)threadIdx.x < heads) s_first[threadIdx.x] = pr.first_rows ? pr.first_rows[threadIdx.x] : 0;
  }
  __syncthreads();
  long long kept = s_off[heads];
  if (kept > pr.capacity) kept = pr.capacity;
  const uint4* __restrict__ k = static_cast<const uint4*>(pr.k_src);
  const uint4* __restrict__ v = static_cast<const uint4*>(pr.v_src);
  uint4* __restrict__ k_out = reinterpret_cast<uint4*>(a.k);
  uint4* __restrict__ v_out = reinterpret_cast<uint4*>(a.v);
  const int c = threadIdx.x % LPR;
  for (long long t = (long long)blockIdx.x * kRowsPerBlock + threadIdx.x / LPR; t < kept;
       t += (long long)gridDim.x * kRowsPerBlock) {
    int g = 0;
    while (g + 1 < heads && t >= s_off[g + 1]) ++g;
    const long long src = (long long)pr.kept_idx[t], len = s_src[g + 1] - s_src[g];
    const long long row = (long long)s_first[g] + t - s_off[g];
    const long long block = row >> a.page_shift;
    // a source row outside the head's segment (or, packed, its pool) and a row outside the head's table are no rows
    if (src < 0 || src >= len || s_src[g] < 0 || (pr.src_offsets != nullptr && s_src[g + 1] > pr.src_rows)) continue;
    if (row < 0 || block >= a.max_blocks) continue;
    const long long page = (long long)pr.block_table[(long long)g * a.max_blocks + block];
    if (page < 0 || page >= a.n_pages) continue;
    const long long in = s_src[g] + src;
    const long long slot = (page << a.page_shift) + (row & ((1 << a.page_shift) - 1));
    const uint4 kv = k[in * LPR + c], vv = v[in * LPR + c];
    k_out[slot * LPR + c] = kv;
    v_out[slot * LPR + c] = vv;
    if (a.pos != nullptr && c == 0) a.pos[slot] = pr.pos_src ? pr.pos_src[in] : (int32_t)src;
  }
}

}  // namespace

int32_t launch_compact_paged(const lava_layer_desc& d, int n_problems, const lava_paged_compact_problem* problems,
                             const lava_page_pool& pool, hipStream_t s) {
  const int lpr = d.head_dim * (d.dtype == LAVA_BF16 ? 2 : 4) / 16;
  const int rows_per_block = kGatherThreads / lpr;
  PagedBatch a;
  a.k = static_cast<char*>(pool.k);
  a.v = static_cast<char*>(pool.v);
  a.pos = pool.pos;
  a.n_pages = pool.n_pages;
  a.max_blocks = pool.max_blocks;
  a.page_shift = __builtin_ctz((unsigned)pool.page_rows);
  a.n_heads = d.n_kv_heads;
  for (int first = 0; first < n_problems; first += kMaxSelProblems) {
    const int count = n_problems - first < kMaxSelProblems ? n_problems - first : kMaxSelProblems;
    int64_t widest = 0;
    for (int i = 0; i < count; ++i) {
      a.p[i] = problems[first + i];
      if (a.p[i].capacity > widest) widest = a.p[i].capacity;
    }
    if (widest == 0) continue;
    int64_t bx = (widest + rows_per_block - 1) / rows_per_block;
    if (bx > 1024) bx = 1024;
    ProfScope ps(KID_COMPACT, s);
    const dim3 grid((unsigned)bx, count), block(kGatherThreads);
    switch (lpr) {
      case 8: hipLaunchKernelGGL(compact_paged_kernel<8>, grid, block, 0, s, a); break;
      case 16: hipLaunchKernelGGL(compact_paged_kernel<16>, grid, block, 0, s, a); break;
      case 32: hipLaunchKernelGGL(compact_paged_kernel<32>, grid, block, 0, s, a); break;
      default: return LAVA_ERR_SHAPE;
    }
    const int32_t st = launch_status();
    if (st != LAVA_OK) return st;
  }
  return LAVA_OK;
}

}  // namespace lava
