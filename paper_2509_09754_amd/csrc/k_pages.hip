// Pages of the paged cache: block tables and slot maps of a step, and the gather of an eviction's
// survivors into pages.
//
// A step's tables are exclusive sums over the heads in order: head i needs ceil((old + add) / P) - ceil(old / P)
// pages and pops them behind those of the heads before it.  Everything else follows from the sums: which page a
// new block gets is one look-up in the stack, which slot a new row has is one look-up in the stack or the table.
#include "common.h"

namespace lava {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;

// What the plan leaves in the workspace for the fill.
struct PlanHeader {
  int error;             // LAVA_PAGES_* bits; 0: the step is carried out
  int top;               // pages on the stack once those given back are on it
  int tokens;            // new tokens of all sequences
  int pad;
};
struct PlanLayout {
  size_t off_old;        // int [heads]      rows every head starts the step with (0 where it is over)
  size_t off_need;       // int [heads + 1]  pages needed by the heads before
  size_t off_back;       // int [heads + 1]  pages given back by the heads before
  size_t off_tok;        // int [batch + 1]  new tokens of the sequences before
  size_t off_pos;        // int [batch]      position of every sequence's first new token
  size_t bytes;
};
__host__ __device__ inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
__host__ __device__ inline PlanLayout plan_layout(int batch, int heads) {
  PlanLayout l;
  l.off_old = 256;
  l.off_need = l.off_old + up256((size_t)heads * 4);
  l.off_back = l.off_need + up256((size_t)(heads + 1) * 4);
  l.off_tok = l.off_back + up256((size_t)(heads + 1) * 4);
  l.off_pos = l.off_tok + up256((size_t)(batch + 1) * 4);
  l.bytes = l.off_pos + up256((size_t)batch * 4);
  return l;
}

__device__ __forceinline__ long long shfl_up64(long long x, int d) {
  const int lo = __shfl_up((int)(unsigned int)x, d), hi = __shfl_up((int)(x >> 32), d);
  return ((long long)hi << 32) | (unsigned int)lo;
}

// Exclusive sum over the workgroup's threads; *total: the sum over all.
__device__ __forceinline__ long long block_scan(long long x, long long* s_part, long long* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  long long incl = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long long y = shfl_up64(incl, d);
    if (lane >= d) incl += y;
  }
  if (lane == 63) s_part[wave] = incl;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const long long p = s_part[w];
    if (w < wave) before += p;
    all += p;
  }
  __syncthreads();
  *total = all;
  return before + incl - x;
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

// The sums, by one workgroup.
__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const PageTablesArgs a) {
  __shared__ long long s_part[kPlanWaves];
  __shared__ int s_error;
  const int heads = a.batch * a.heads;
  const PlanLayout l = plan_layout(a.batch, heads);
  char* ws = static_cast<char*>(a.ws);
  int* w_old = reinterpret_cast<int*>(ws + l.off_old);
  int* w_need = reinterpret_cast<int*>(ws + l.off_need);
  int* w_back = reinterpret_cast<int*>(ws + l.off_back);
  int* w_tok = reinterpret_cast<int*>(ws + l.off_tok);
  int* w_pos = reinterpret_cast<int*>(ws + l.off_pos);
  if (threadIdx.x == 0) s_error = 0;
  __syncthreads();
  int error = 0;
  long long need = 0, back = 0, tokens = 0;
  for (int h0 = 0; h0 < heads; h0 += kPlanThreads) {
    const int hb = h0 + (int)threadIdx.x;
    HeadStep h = {0, 0, 0, 0, 0};
    if (hb < heads) h = head_step(a, hb);
    error |= h.error;
    long long t_need, t_back;
    const long long n0 = block_scan(h.need, s_part, &t_need), b0 = block_scan(h.back, s_part, &t_back);
    if (hb < heads) {
      w_old[hb] = h.old;
      w_need[hb] = (int)(need + n0);       // read only if the step is carried out: the sum is below 2^31 then
      w_back[hb] = (int)(back + b0);
    }
    need += t_need;
    back += t_back;
  }
  for (int s0 = 0; s0 < a.batch; s0 += kPlanThreads) {
    const int b = s0 + (int)threadIdx.x;
    int n = 0;
    if (b < a.batch) {
      n = a.n_new != nullptr ? a.n_new[b] : 0;
      const bool over = a.release != nullptr && a.release[b] != 0;
      const int pos = over ? 0 : a.st.seq_pos[b];
      if (n < 0 || pos < 0 || (long long)pos + n >= (long long)1 << 31) {
        error |= LAVA_PAGES_INVALID;
        n = 0;
      }
      w_pos[b] = pos;
    }
    long long t_tok;
    const long long t0 = block_scan(n, s_part, &t_tok);
    if (b < a.batch) w_tok[b] = (int)(tokens + t0);
    tokens += t_tok;
  }
  const long long free_pages = a.st.n_free[0];
  if (free_pages < 0 || free_pages + back > a.n_pages) error |= LAVA_PAGES_INVALID;
  else if (need > free_pages + back) error |= LAVA_PAGES_EXHAUSTED;
  if (a.slots != nullptr || a.positions != nullptr) {
    if (tokens > a.max_tokens) error |= LAVA_PAGES_TOKENS;
  }
  if (error != 0) atomicOr(&s_error, error);
  __syncthreads();
  if (threadIdx.x == 0) {
    w_need[heads] = (int)need;
    w_back[heads] = (int)back;
    w_tok[a.batch] = (int)tokens;
    PlanHeader* hd = reinterpret_cast<PlanHeader*>(ws);
    hd->error = s_error;
    hd->top = (int)(free_pages + back);
    hd->tokens = (int)tokens;
    if (s_error != 0 && a.st.error != nullptr) atomicOr(a.st.error, s_error);
  }
}

// Pages of the sequences that are over, onto the stack: a wavefront per head.
__global__ void __launch_bounds__(256) page_return_kernel(const PageTablesArgs a) {
  const char* ws = static_cast<const char*>(a.ws);
  if (reinterpret_cast<const PlanHeader*>(ws)->error != 0) return;
  const int heads = a.batch * a.heads;
  const PlanLayout l = plan_layout(a.batch, heads);
  const int* w_back = reinterpret_cast<const int*>(ws + l.off_back);
  const int lane = threadIdx.x & 63;
  const int free_pages = reinterpret_cast<const PlanHeader*>(ws)->top - w_back[heads];
  for (int hb = blockIdx.x * 4 + (threadIdx.x >> 6); hb < heads; hb += gridDim.x * 4) {
    const int first = w_back[hb], n = w_back[hb + 1] - first;
    const int* table = a.st.block_table + (long long)hb * a.max_blocks;
    for (int j = lane; j < n; j += 64) a.st.free_pages[free_pages + first + j] = table[j];
  }
}

// Tables, counts, slots and positions.  The first `head_wgs` workgroups take the heads (a wavefront each), the others
// the tokens.
__global__ void __launch_bounds__(256) page_fill_kernel(const PageTablesArgs a, const int head_wgs) {
  const char* ws = static_cast<const char*>(a.ws);
  const PlanHeader hd = *reinterpret_cast<const PlanHeader*>(ws);
  const int heads = a.batch * a.heads;
  const PlanLayout l = plan_layout(a.batch, heads);
  const int* w_old = reinterpret_cast<const int*>(ws + l.off_old);
  const int* w_need = reinterpret_cast<const int*>(ws + l.off_need);
  const int* w_tok = reinterpret_cast<const int*>(ws + l.off_tok);
  const int* w_pos = reinterpret_cast<const int*>(ws + l.off_pos);
  const int mask = (1 << a.page_shift) - 1;
  const int lane = threadIdx.x & 63;
  if ((int)blockIdx.x < head_wgs) {
    for (int hb = blockIdx.x * 4 + (threadIdx.x >> 6); hb < heads; hb += head_wgs * 4) {
      const int b = hb / a.heads;
      if (hd.error != 0) {
        if (lane == 0) a.st.head_rows_out[hb] = a.st.head_rows[hb];
        continue;
      }
      const int old = w_old[hb], start = w_need[hb], need = w_need[hb + 1] - start;
      const int first = (old + mask) >> a.page_shift;
      int* table = a.st.block_table + (long long)hb * a.max_blocks + first;
      for (int j = lane; j < need; j += 64) table[j] = a.st.free_pages[hd.top - 1 - start - j];
      if (lane == 0) {
        const int add = a.head_counts != nullptr ? a.head_counts[hb] : a.n_new != nullptr ? a.n_new[b] : 0;
        a.st.head_rows_out[hb] = old + add;
      }
    }
    for (int b = blockIdx.x * 256 + (int)threadIdx.x; b < a.batch; b += head_wgs * 256) {
      const int pos = a.st.seq_pos[b], n = a.n_new != nullptr ? a.n_new[b] : 0;
      const bool over = a.release != nullptr && a.release[b] != 0;
      a.st.seq_pos_out[b] = hd.error != 0 ? pos : (over ? 0 : pos) + n;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0)
      a.st.n_free_out[0] = hd.error != 0 ? a.st.n_free[0] : hd.top - w_need[heads];
    return;
  }
  const int wg = blockIdx.x - head_wgs, wgs = gridDim.x - head_wgs;
  const long long all = a.max_tokens * a.heads, real = hd.error != 0 ? 0 : (long long)hd.tokens * a.heads;
  for (long long e = (long long)wg * 256 + (int)threadIdx.x; e < all; e += (long long)wgs * 256) {
    const int t = (int)(e / a.heads), g = (int)(e - (long long)t * a.heads);
    if (e >= real) {
      if (a.slots != nullptr) a.slots[e] = -1;
      if (a.positions != nullptr && g == 0) a.positions[t] = -1;
      continue;
    }
    int lo = 0, hi = a.batch - 1;                             // the sequence: the last one that starts at or before t
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (w_tok[mid] <= t) lo = mid; else hi = mid - 1;
    }
    const int i = t - w_tok[lo];
    if (a.positions != nullptr && g == 0) a.positions[t] = w_pos[lo] + i;
    if (a.slots == nullptr) continue;
    const int hb = lo * a.heads + g, old = w_old[hb], r = old + i;
    const int block = r >> a.page_shift, first = (old + mask) >> a.page_shift;
    const int page = block < first ? a.st.block_table[(long long)hb * a.max_blocks + block]
                                   : a.st.free_pages[hd.top - 1 - w_need[hb] - (block - first)];
    a.slots[e] = ((long long)page << a.page_shift) + (r & mask);
  }
}

}  // namespace

size_t page_tables_bytes(int32_t batch, int32_t n_kv_heads) { return plan_layout(batch, batch * n_kv_heads).bytes; }

int32_t launch_page_tables(const PageTablesArgs& a, hipStream_t s) {
  {
    ProfScope ps(KID_PAGE_PLAN, s);
    hipLaunchKernelGGL(page_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
  }
  int32_t st = launch_status();
  if (st != LAVA_OK) return st;
  const long long heads = (long long)a.batch * a.heads;
  long long head_wgs = (heads + 3) / 4, wgs = 0;
  if (head_wgs > 2048) head_wgs = 2048;
  if (a.release != nullptr) {
    ProfScope ps(KID_PAGE_FILL, s);
    hipLaunchKernelGGL(page_return_kernel, dim3((unsigned)head_wgs), dim3(256), 0, s, a);
    st = launch_status();
    if (st != LAVA_OK) return st;
  }
  if (a.max_tokens > 0) {
    wgs = (a.max_tokens * a.heads + 255) / 256;
    if (wgs > 4096) wgs = 4096;
  }
  ProfScope ps(KID_PAGE_FILL, s);
  hipLaunchKernelGGL(page_fill_kernel, dim3((unsigned)(head_wgs + wgs)), dim3(256), 0, s, a, (int)head_wgs);
  return launch_status();
}

// ------------------------------------------------------------------------------------------
// The gather of an eviction's survivors into pages: bound by HBM, 4 * d_h * elem bytes a row.  A row is
// moved by (row bytes / 16) lanes; the workgroups of a problem walk over its survivors.
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
