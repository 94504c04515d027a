// Sequences that become copies of others, lose rows or end, over pages that sequences share.
//
// A new head takes rows of an old one: all of them (fork) or the ascending list r_0 < r_1 < .. that a selection keeps (compact).  With
// `same` the number of leading t with r_t = t, the first floor(same / P) blocks are blocks of the old table, and so is the
// last one where the head keeps all rows of a last page that was not full and is the copy that goes on with it.  The blocks
// behind them go to fresh pages, whose rows are copied.  A page is free afterwards if no new table names it.
//
// Who holds a page is found out by marking, two words a page: a new table's leading blocks store `alive`, an old table's blocks that
// do not stay in their places take the minimum with 1 + the head's number in `first`.  A page that is not alive was first named by head
// first - 1, which gives it back, so that the stack's order does not depend on the order of the marks.
//
// Each step needs all of what the one before found: clear the marks; mark, and sum the fresh pages over the heads (a
// wavefront a head, partial sums by workgroup); count what goes back, and take the fresh pages off the stack; write tables,
// counts, stack, and copy rows, the fresh pages' rows in one line that the workgroups share evenly.  What the last step
// reads of buffers that it also writes was set aside before.  The first three are one launch of one workgroup where tables are few
// and short (kOneEntries), which clears only the words of pages that are named.
//
// Bound by the chain of launches and of look-ups in each for a beam step (one layer of eight beams of 4096 tokens: 7.3 us by one workgroup, 5.8 of
// rows; 32 layers of 16 beams: 2.9, 6.0, 5.0 and 16 for 47 MB), by HBM for many rows (48 caches evicted in 32 bits, 254 MB:
// rows 60 us, 4.3 TB/s, marks 21).  An entry that names the page it named before is no candidate for going back: with
// atomics for the pages that all beams share the second launch of the 32 layers took 8.5 us.
#include "common.h"
#include "decode_parts.h"
#include "tile_ring.h"
#include "xblock.h"

namespace lava {

namespace {

constexpr int kChangeWaves = 4, kChangeThreads = kChangeWaves * 64;   // of a workgroup that sums over heads
constexpr int kMostGroups = 1024;             // workgroups of a launch that sums over heads
constexpr unsigned int kNoHolder = 0xffffffffu;

struct ChangeHeader {
  int error;                                  // LAVA_PAGES_* bits
  int n_free, fresh;                          // free pages before, pages taken
};

struct __attribute__((aligned(16))) HeadPlan {
  int n, stay;                                // rows, and leading blocks that stay, after the call
  int from, old;                              // head that it comes from (-1: none), rows that one held
  long long list;                             // first entry of its list in the sequence's, -1: it keeps all rows
  int fresh_at, back_at;                      // pages taken by the heads before it; given back by those (of its workgroup) before it
};

struct ChangeArgs {
  PageChangeArgs p;
  ChangeHeader* head;
  int *fresh_total, *back_total;              // [kMostGroups] of a workgroup's heads
  int* seq_pos;                               // [batch] position after the call
  int* old_rows;                              // [heads]
  HeadPlan* plan;                             // [heads]
  unsigned int *alive, *first;                // [n_pages]
  int *taken, *owner;                         // [n_pages] fresh pages in order, the heads that take them
  int* old_table;                             // [heads][max_blocks] a copy, if the tables change in place
  int heads, per;                             // heads in all, heads a wavefront that sums
  int one;                                    // the marks are one workgroup's
};

struct ChangeLayout {
  size_t off_fresh, off_back, off_pos, off_rows, off_plan, off_alive, off_first, off_taken, off_owner, off_table, bytes;
};
ChangeLayout change_layout(int batch, int n_kv_heads, int max_blocks, long long n_pages) {
  ChangeLayout l;
  const size_t heads = (size_t)batch * n_kv_heads, pages = align_up((size_t)n_pages * 4);
  l.off_fresh = align_up(sizeof(ChangeHeader));
  l.off_back = l.off_fresh + align_up(kMostGroups * 4);
  l.off_pos = l.off_back + align_up(kMostGroups * 4);
  l.off_rows = l.off_pos + align_up((size_t)batch * 4);
  l.off_plan = l.off_rows + align_up(heads * 4);
  l.off_alive = l.off_plan + align_up(heads * sizeof(HeadPlan));
  l.off_first = l.off_alive + pages;
  l.off_taken = l.off_first + pages;
  l.off_owner = l.off_taken + pages;
  l.off_table = l.off_owner + pages;
  l.bytes = l.off_table + align_up(heads * max_blocks * 4);
  return l;
}

__device__ __forceinline__ bool is_page(const PageChangeArgs& p, int page) { return page >= 0 && page < p.n_pages; }

// Rows of a head with that count, 0 where it is out of range.
__device__ __forceinline__ int rows_of(const PageChangeArgs& p, int rows) {
  return rows < 0 || rows > (long long)p.max_blocks << p.page_shift ? 0 : rows;
}

__device__ __forceinline__ int blocks_of(const PageChangeArgs& p, int rows) {
  return (int)(((long long)rows + (1 << p.page_shift) - 1) >> p.page_shift);
}

// Does sequence b go on with the last pages of sequence s, which it is made of?  A wavefront's question.
__device__ __forceinline__ bool is_keeper(const PageChangeArgs& p, int b, int s) {
  if (p.source == nullptr || s == b) return true;
  if (s < 0) return false;
  const int lane = threadIdx.x & 63, of_s = p.source[s];
  for (int c0 = 0; c0 < b; c0 += 512) {
    bool same = false;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int c = c0 + 64 * u + lane;
      same |= c < b && p.source[c < b ? c : b] == s;
    }
    if (__ballot(same) != 0ull) return false;
  }
  return of_s != s;
}

// The first t in [0, n) with list[t] != t, n if there is none; the list ascends.
__device__ __forceinline__ int leading_same(const int* list, int n) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64, probes = (hi - lo + step - 1) / step;
    const int t = lo + lane * step;
    const unsigned long long off = __ballot(lane < probes && list[lane < probes ? t : lo] != t);
    if (off == 0ull) {
      lo += (probes - 1) * step + 1;
    } else {
      const int f = __builtin_ctzll(off);
      if (f == 0) return lo;
      hi = lo + f * step;
      lo += (f - 1) * step + 1;
    }
  }
  return lo;
}

constexpr int kLooks = 4;                     // look-ups of a thread at a time

// What head h keeps, and its marks; returns the fresh pages it needs.  A wavefront's work; error bits are or-ed to `error`.
// The kernel takes as long as its chain of look-ups, so the first blocks of both tables are loaded before it is known how
// many count, and who keeps a last page is found out while the counts are on their way.
__device__ __forceinline__ int mark_head(const ChangeArgs& a, int h, int& error) {
  const PageChangeArgs& p = a.p;
  const int lane = threadIdx.x & 63, G = p.heads, P = 1 << p.page_shift, b = h / G, g = h - b * G;
  const int* mine = p.st.block_table + (long long)h * p.max_blocks;
  const int mine_first = mine[lane < p.max_blocks ? lane : 0], held = p.st.head_rows[h];
  int s = p.source != nullptr ? p.source[b] : b;
  if (s < -1 || s >= p.batch) error |= LAVA_PAGES_INVALID, s = -1;
  const int* from = p.st.block_table + ((long long)(s >= 0 ? s : b) * G + g) * p.max_blocks;
  const int from_first = from[lane < p.max_blocks ? lane : 0], held_from = p.st.head_rows[(s >= 0 ? s : b) * G + g];
  const int from_pos = p.st.seq_pos[s >= 0 ? s : b];
  const bool keeper = is_keeper(p, b, s);
  const int rows = rows_of(p, held), nb_old = blocks_of(p, rows), old = s >= 0 ? rows_of(p, held_from) : 0;
  if (held != rows) error |= LAVA_PAGES_INVALID;
  int n = old, same = old;
  long long begin = -1;
  if (p.head_counts != nullptr && (p.evict == nullptr || p.evict[b] != 0)) {
    int count = 0;
    bool bad = false;
    if (lane < G) {
      count = p.head_counts[(long long)b * G + lane];
      bad = count < 0 || count > p.st.head_rows[b * G + lane];
    }
    long long all = 0, before = 0;
    for (int i = 0; i < G; ++i) {
      const int c = (int)lane_value((unsigned int)count, i);
      before += i < g ? c : 0;
      all += c;
    }
    if (__ballot(bad) != 0ull || all > p.kept_capacity) {
      error |= LAVA_PAGES_INVALID;
      n = same = 0;
    } else {
      n = (int)lane_value((unsigned int)count, g);
      begin = before;
      same = leading_same(p.kept_idx + (long long)b * p.kept_capacity + begin, n);
    }
  }
  int stay = same >> p.page_shift;
  if ((n & (P - 1)) != 0 && same >= n && (old & (P - 1)) != 0 && n >> p.page_shift == old >> p.page_shift && keeper) ++stay;
  if (s >= 0) {
    for (int j0 = lane; j0 < stay; j0 += 64 * kLooks) {
      int page[kLooks];
#pragma unroll
      for (int u = 0; u < kLooks; ++u) page[u] = j0 + 64 * u < 64 ? from_first : j0 + 64 * u < stay ? from[j0 + 64 * u] : 0;
#pragma unroll
      for (int u = 0; u < kLooks; ++u) {
        if (j0 + 64 * u >= stay) continue;
        if (!is_page(p, page[u])) error |= LAVA_PAGES_INVALID;
        else a.alive[page[u]] = 1u;
      }
    }
  }
  const int kept = s == b ? stay : 0;                          // leading blocks that this head marked itself
  const int beside = s >= 0 ? stay : 0;                        // where it may have: the two tables name the same pages, as a prompt's beams do
  for (int j0 = lane; j0 < nb_old; j0 += 64 * kLooks) {
    int page[kLooks], other[kLooks];
#pragma unroll
    for (int u = 0; u < kLooks; ++u) {
      const int j = j0 + 64 * u;
      page[u] = j < 64 ? mine_first : j < nb_old && (j >= kept || a.old_table != nullptr) ? mine[j] : 0;
      other[u] = j >= beside ? -1 : j < 64 ? from_first : j < nb_old ? from[j] : -1;
    }
#pragma unroll
    for (int u = 0; u < kLooks; ++u) {
      const int j = j0 + 64 * u;
      if (j >= nb_old) continue;
      if (a.old_table != nullptr) a.old_table[(long long)h * p.max_blocks + j] = page[u];
      if (j < kept) continue;
      if (!is_page(p, page[u])) error |= LAVA_PAGES_INVALID;
      else if (page[u] != other[u]) __hip_atomic_fetch_min(&a.first[page[u]], 1u + (unsigned int)h, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  if (lane == 0) {
    a.old_rows[h] = rows;
    HeadPlan& x = a.plan[h];
    x.n = n;
    x.stay = stay;
    x.from = s >= 0 ? s * G + g : -1;
    x.old = old;
    x.list = begin;
    if (g == 0) a.seq_pos[b] = s >= 0 ? from_pos : 0;
  }
  return blocks_of(p, n) - stay;
}

// Pages that head h gives back.  `use(page, how many before it)` for each, in the order of the blocks; a wavefront's work.
template <typename F>
__device__ __forceinline__ int for_each_gone(const ChangeArgs& a, int h, const int* table, F use) {
  const int lane = threadIdx.x & 63, first_page = table[lane < a.p.max_blocks ? lane : 0], nb_old = blocks_of(a.p, a.old_rows[h]);
  int n = 0;
  for (int j0 = a.plan[h].from == h ? a.plan[h].stay & ~63 : 0; j0 < nb_old; j0 += 64 * kLooks) {   // (what stays is alive)
    int page[kLooks];
    unsigned int first[kLooks], alive[kLooks];
#pragma unroll
    for (int u = 0; u < kLooks; ++u) {
      const int j = j0 + 64 * u + lane;
      page[u] = j >= nb_old ? -1 : j0 + 64 * u == 0 ? first_page : table[j];
    }
#pragma unroll
    for (int u = 0; u < kLooks; ++u) {
      const bool there = is_page(a.p, page[u]);
      first[u] = there ? a.first[page[u]] : kNoHolder;
      alive[u] = there ? a.alive[page[u]] : 1u;
    }
#pragma unroll
    for (int u = 0; u < kLooks; ++u) {
      const bool gone = first[u] == 1u + (unsigned int)h && alive[u] == 0u;
      const unsigned long long all = __ballot(gone);
      if (gone) use(page[u], n + __popcll(all & ((1ull << lane) - 1ull)));
      n += __popcll(all);
    }
  }
  return n;
}

// The sum of the wavefronts' values (y) and of those before this one (x).
__device__ __forceinline__ int2 sums_of_group(int* s_wave, int mine) {
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) s_wave[wave] = mine;
  __syncthreads();
  int2 r = make_int2(0, 0);
#pragma unroll
  for (int w = 0; w < kChangeWaves; ++w) {
    r.x += w < wave ? s_wave[w] : 0;
    r.y += s_wave[w];
  }
  __syncthreads();
  return r;
}

// The fresh pages, off the stack: every `step`th from `from` on.  Returns error bits.
__device__ __forceinline__ int take_pages(const ChangeArgs& a, int n_free, int fresh, int from, int step) {
  if (n_free < 0 || n_free > a.p.n_pages || fresh > n_free) return 0;    // found out again when tables are written
  int error = 0;
  for (int k = from; k < fresh; k += step) {
    const int page = a.p.st.free_pages[n_free - 1 - k];
    if (!is_page(a.p, page)) error = LAVA_PAGES_INVALID;
    a.taken[k] = page;
  }
  return error;
}

// ---------------------------------------------------------------- 1: clear
__global__ void __launch_bounds__(256) change_begin_kernel(const ChangeArgs a) {
  if (blockIdx.x == 0 && threadIdx.x == 0) a.head->error = 0;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < a.p.n_pages; i += (long long)gridDim.x * 256) {
    a.alive[i] = 0u;
    a.first[i] = kNoHolder;
  }
}

// ---------------------------------------------------------------- 2: what every head keeps; marks; sums of the fresh pages
__global__ void __launch_bounds__(kChangeThreads) change_mark_kernel(const ChangeArgs a) {
  __shared__ int s_wave[kChangeWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int h0 = (blockIdx.x * kChangeWaves + wave) * a.per, h1 = h0 + a.per < a.heads ? h0 + a.per : a.heads;
  int error = 0, sum = 0;
  for (int h = h0; h < h1; ++h) {
    const int fresh = mark_head(a, h, error);
    if (lane == 0 && a.per > 1) a.plan[h].fresh_at = sum;
    sum += fresh;
  }
  if (error != 0) atomicOr(&a.head->error, error);
  const int2 all = sums_of_group(s_wave, sum);
  if (lane == 0)
    for (int h = h0; h < h1; ++h) a.plan[h].fresh_at = all.x + (a.per > 1 ? a.plan[h].fresh_at : 0);
  if (threadIdx.x == 0) a.fresh_total[blockIdx.x] = all.y;
}

// ---------------------------------------------------------------- 3: sums of what goes back; the fresh pages
__global__ void __launch_bounds__(kChangeThreads) change_count_kernel(const ChangeArgs a) {
  __shared__ int s_wave[kChangeWaves], s_before[kChangeWaves], s_fresh[kChangeWaves];
  const PageChangeArgs& p = a.p;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int h0 = (blockIdx.x * kChangeWaves + wave) * a.per, h1 = h0 + a.per < a.heads ? h0 + a.per : a.heads;
  // fresh pages of the workgroups before this one, of all; they are on their way while the heads' pages are looked up
  constexpr int kEach = kMostGroups / kChangeThreads;
  int fresh_of[kEach], before = 0, fresh = 0, sum = 0;
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const unsigned int i = threadIdx.x + u * kChangeThreads;
    fresh_of[u] = i < gridDim.x ? a.fresh_total[i] : 0;
  }
  const int n_free = p.st.n_free[0];
  for (int h = h0; h < h1; ++h) {
    const int n = for_each_gone(a, h, p.st.block_table + (long long)h * p.max_blocks, [](int, int) {});
    if (lane == 0 && a.per > 1) a.plan[h].back_at = sum;
    sum += n;
  }
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    before += threadIdx.x + u * kChangeThreads < blockIdx.x ? fresh_of[u] : 0;
    fresh += fresh_of[u];
  }
  before = (int)lane_value(wave_incl((unsigned int)before), 63);
  fresh = (int)lane_value(wave_incl((unsigned int)fresh), 63);
  if (lane == 0) {
    s_before[wave] = before;
    s_fresh[wave] = fresh;
  }
  __syncthreads();
  before = fresh = 0;
#pragma unroll
  for (int w = 0; w < kChangeWaves; ++w) {
    before += s_before[w];
    fresh += s_fresh[w];
  }
  const bool enough = n_free >= 0 && n_free <= p.n_pages && fresh <= n_free;
  for (int h = h0; h < h1; ++h) {
    const int at = a.plan[h].fresh_at + before, need = blocks_of(p, a.plan[h].n) - a.plan[h].stay;
    for (int j = lane; enough && j < need; j += 64) a.owner[at + j] = h;
    if (lane == 0) a.plan[h].fresh_at = at;
  }
  const int2 all = sums_of_group(s_wave, sum);
  if (lane == 0)
    for (int h = h0; h < h1; ++h) a.plan[h].back_at = all.x + (a.per > 1 ? a.plan[h].back_at : 0);
  if (threadIdx.x == 0) {
    a.back_total[blockIdx.x] = all.y;
    if (blockIdx.x == 0) {
      a.head->n_free = n_free;
      a.head->fresh = fresh;
    }
  }
  const int error = take_pages(a, n_free, fresh, blockIdx.x * kChangeThreads + threadIdx.x, gridDim.x * kChangeThreads);
  if (error != 0) atomicOr(&a.head->error, error);
}

// ---------------------------------------------------------------- 1 to 3 by one workgroup
// One launch instead of three: eight beams of one layer 7.3 us instead of 14, a wavefront a head in series 25.
// Every thread has up to kOnePer entries of the tables, whose look-ups are independent of each other.  A list's blocks stay as long as
// their last rows are where they were, since it ascends.
constexpr int kOneThreads = 1024, kOneHeads = 256, kOnePer = 8, kOneEntries = kOnePer * kOneThreads;
__global__ void __launch_bounds__(kOneThreads) change_one_kernel(const ChangeArgs a) {
  __shared__ int s_rows[kOneHeads], s_count[kOneHeads], s_source[kOneHeads], s_n[kOneHeads], s_stay[kOneHeads], s_from[kOneHeads];
  __shared__ int s_need[kOneHeads], s_back[kOneHeads], s_whole[kOneHeads], s_error, s_total[2];
  __shared__ long long s_list[kOneHeads];
  const PageChangeArgs& p = a.p;
  const int lane = threadIdx.x & 63, h = threadIdx.x, G = p.heads, P = 1 << p.page_shift, W = p.max_blocks, heads = a.heads;
  const bool is_head = h < heads;
  const int b = is_head ? h / G : 0, g = h - b * G;
  if (threadIdx.x == 0) s_error = 0;
  const int n_free = p.st.n_free[0];
  int error = 0, entry_page[kOnePer], entry_head[kOnePer], entry_block[kOnePer];
  const double inv_w = 1.0 / (double)W;                        // e / W: half an entry off the border, so the product is exact enough
#pragma unroll
  for (int u = 0; u < kOnePer; ++u) {
    const int e = u * kOneThreads + (int)threadIdx.x;
    entry_head[u] = e < heads * W ? (int)(((double)e + 0.5) * inv_w) : -1;
    entry_block[u] = e - entry_head[u] * W;
    entry_page[u] = entry_head[u] >= 0 ? p.st.block_table[e] : -1;   // behind a head's last block whatever is there: not used
  }
  if (is_head) {
    const int held = p.st.head_rows[h], rows = rows_of(p, held);
    if (held != rows) error = LAVA_PAGES_INVALID;
    s_rows[h] = rows;
    s_count[h] = p.head_counts != nullptr ? p.head_counts[h] : 0;
    s_back[h] = 0;
    if (h < p.batch) {
      int s = p.source != nullptr ? p.source[h] : h;
      if (s < -1 || s >= p.batch) error = LAVA_PAGES_INVALID, s = -1;
      s_source[h] = s;
    }
  }
  __syncthreads();
  int n = 0, old = 0, s = -1;
  long long begin = -1;
  bool keeper = false;
  if (is_head) {
    s = s_source[b];
    old = s >= 0 ? s_rows[s * G + g] : 0;
    n = old;
    keeper = s == b || (s >= 0 && s_source[s] != s);
    for (int c = 0; s != b && c < b; ++c) keeper = keeper && s_source[c] != s;
    if (p.head_counts != nullptr && (p.evict == nullptr || p.evict[b] != 0)) {
      long long all = 0, before = 0;
      bool bad = false;
      for (int i = 0; i < G; ++i) {
        const int c = s_count[b * G + i];
        bad |= c < 0 || c > s_rows[b * G + i];
        before += i < g ? c : 0;
        all += c;
      }
      bad |= all > p.kept_capacity;
      if (bad) error = LAVA_PAGES_INVALID;
      n = bad ? 0 : s_count[h];
      begin = before;
    }
    s_n[h] = n;
    s_from[h] = s >= 0 ? s * G + g : -1;
    s_list[h] = begin >= 0 ? (long long)b * p.kept_capacity + begin : -1;
    s_stay[h] = begin >= 0 ? 0 : n >> p.page_shift;
    s_whole[h] = begin < 0 || (n > 0 && p.kept_idx[(long long)b * p.kept_capacity + begin + n - 1] == n - 1) ? 1 : 0;
    a.old_rows[h] = s_rows[h];
    if (g == 0) a.seq_pos[b] = s >= 0 ? p.st.seq_pos[s] : 0;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kOnePer; ++u) {
    const int x = entry_head[u], j = entry_block[u], page = entry_page[u];
    if (x < 0) continue;
    if (j < blocks_of(p, s_rows[x])) {
      if (a.old_table != nullptr) a.old_table[x * W + j] = page;
      if (is_page(p, page)) {
        st_dev(&a.alive[page], 0u);
        st_dev(&a.first[page], kNoHolder);
      } else {
        error = LAVA_PAGES_INVALID;
      }
    } else {
      entry_page[u] = -1;
    }
    if (s_list[x] >= 0 && (long long)(j + 1) << p.page_shift <= s_n[x]) {
      const int last = ((j + 1) << p.page_shift) - 1;
      if (p.kept_idx[s_list[x] + last] == last) atomicAdd(&s_stay[x], 1);
    }
  }
  drain_vmem();
  __syncthreads();
  if (is_head) {
    if ((n & (P - 1)) != 0 && s_whole[h] != 0 && (old & (P - 1)) != 0 && n >> p.page_shift == old >> p.page_shift && keeper) s_stay[h] += 1;
    s_need[h] = blocks_of(p, n) - s_stay[h];
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kOnePer; ++u) {
    const int x = entry_head[u], j = entry_block[u], page = entry_page[u];
    if (x < 0) continue;
    const int from = s_from[x], stay = s_stay[x];
    int keeps = -1;
    if (from >= 0 && j < stay) {
      keeps = from == x ? page : p.st.block_table[from * W + j];
      if (is_page(p, keeps)) st_dev(&a.alive[keeps], 1u);
    }
    if (is_page(p, page) && keeps != page)
      __hip_atomic_fetch_min(&a.first[page], 1u + (unsigned int)x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  drain_vmem();
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kOnePer; ++u) {
    const int x = entry_head[u], page = entry_page[u];
    if (x < 0 || !is_page(p, page) || (s_from[x] == x && entry_block[u] < s_stay[x])) continue;
    if (ld_dev(&a.first[page]) == 1u + (unsigned int)x && ld_dev(&a.alive[page]) == 0u) atomicAdd(&s_back[x], 1);
  }
  __syncthreads();
  if (threadIdx.x < 64) {                                      // exclusive sums over the heads
    int fresh = 0, back = 0;
    for (int h0 = 0; h0 < heads; h0 += 64) {
      const int x = h0 + lane;
      const unsigned int f = x < heads ? (unsigned int)s_need[x] : 0u, r = x < heads ? (unsigned int)s_back[x] : 0u;
      const unsigned int fi = wave_incl(f), ri = wave_incl(r);
      if (x < heads) {
        s_count[x] = fresh + (int)(fi - f);
        s_back[x] = back + (int)(ri - r);
      }
      fresh += (int)lane_value(fi, 63);
      back += (int)lane_value(ri, 63);
    }
    if (lane == 0) {
      s_total[0] = fresh;
      s_total[1] = back;
    }
  }
  __syncthreads();
  const int fresh = s_total[0];
  if (is_head) a.plan[h] = HeadPlan{n, s_stay[h], s_from[h], old, begin, s_count[h], s_back[h]};
  if (n_free >= 0 && n_free <= p.n_pages && fresh <= n_free) {
#pragma unroll
    for (int u = 0; u < kOnePer; ++u) {
      const int x = entry_head[u], j = entry_block[u];
      if (x >= 0 && j < s_need[x]) a.owner[s_count[x] + j] = x;
    }
  }
  error |= take_pages(a, n_free, fresh, threadIdx.x, kOneThreads);
  if (error != 0) atomicOr(&s_error, error);
  __syncthreads();
  if (threadIdx.x == 0) {
    *a.head = ChangeHeader{s_error, n_free, fresh};
    a.back_total[0] = s_total[1];
  }
}

// ---------------------------------------------------------------- 4: tables, counts, stack; rows
constexpr int kApplyThreads = 256, kApplyWaves = kApplyThreads / 64, kMostApply = 4096;
template <int ROWS>                           // rows of a thread at a time
__global__ void __launch_bounds__(kApplyThreads) change_apply_kernel(const ChangeArgs a, int groups) {
  __shared__ int s_before[kMostGroups], s_wave[kApplyWaves];   // pages given back by the groups of heads before each
  const PageChangeArgs& p = a.p;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, G = p.heads, P = 1 << p.page_shift;
  const int first = blockIdx.x * kApplyThreads + threadIdx.x, step = gridDim.x * kApplyThreads;
  const int wave0 = blockIdx.x * kApplyWaves + wave, waves = gridDim.x * kApplyWaves;
  const ChangeHeader head = *a.head;
  int back = 0;                                                // pages given back
  {
    constexpr int kEach = kMostGroups / kApplyThreads;
    int mine[kEach], sum = 0;
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int q = (int)threadIdx.x * kEach + u;
      mine[u] = q < groups ? a.back_total[q] : 0;
    }
#pragma unroll
    for (int u = 0; u < kEach; ++u) sum += mine[u];
    const int incl = (int)wave_incl((unsigned int)sum);
    if (lane == 63) s_wave[wave] = incl;
    __syncthreads();
    int at = incl - sum;
#pragma unroll
    for (int w = 0; w < kApplyWaves; ++w) {
      at += w < wave ? s_wave[w] : 0;
      back += s_wave[w];
    }
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      s_before[threadIdx.x * kEach + u] = at;
      at += mine[u];
    }
    __syncthreads();
  }
  const int n_free = head.n_free;
  int error = head.error;
  if (n_free < 0 || n_free > p.n_pages) error |= LAVA_PAGES_INVALID;
  if (error == 0 && head.fresh > n_free) error = LAVA_PAGES_EXHAUSTED;
  if (error == 0 && (long long)n_free - head.fresh + back > p.n_pages) error = LAVA_PAGES_INVALID;
  const int left = error != 0 ? (n_free < 0 ? 0 : n_free > p.n_pages ? (int)p.n_pages : n_free) : n_free - head.fresh;
  const bool table_apart = p.table_out != p.st.block_table;
  const int* tables = table_apart ? p.st.block_table : a.old_table;
  if (first == 0) {
    p.st.n_free_out[0] = error != 0 ? n_free : left + back;
    if (error != 0 && p.st.error != nullptr) atomicOr(p.st.error, error);
  }
  if (p.free_out != p.st.free_pages)
    for (int i = first; i < left; i += step) p.free_out[i] = p.st.free_pages[i];
  if (error != 0) {                                            // nothing changes
    for (int h = wave0; h < a.heads; h += waves) {
      const long long row = (long long)h * p.max_blocks;
      if (table_apart)
        for (int j = lane; j < blocks_of(p, a.old_rows[h]); j += 64) p.table_out[row + j] = tables[row + j];
      if (lane == 0) {
        p.st.head_rows_out[h] = p.st.head_rows[h];
        if (h % G == 0) p.st.seq_pos_out[h / G] = p.st.seq_pos[h / G];
      }
    }
    return;
  }
  // rows: those of the fresh pages in one line, `per_row` threads a row, ROWS rows of a thread at a time
  const int per_row = p.row_bytes >> 4, rows_a_pass = kApplyThreads / per_row, i = threadIdx.x / per_row, x = threadIdx.x - i * per_row;
  u32x4 *k_out = reinterpret_cast<u32x4*>(p.k), *v_out = reinterpret_cast<u32x4*>(p.v);
  const u32x4 *k_in = k_out, *v_in = v_out;
  const long long pass = (long long)rows_a_pass * ROWS, total = (long long)head.fresh << p.page_shift;
  for (long long t0 = blockIdx.x * pass; t0 < total; t0 += gridDim.x * pass) {
    long long src[ROWS], dst[ROWS];
    bool on[ROWS];
    int owner[ROWS], page[ROWS];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      const long long at = t0 + u * rows_a_pass + i;
      const int k = (int)((at < total ? at : t0) >> p.page_shift);
      owner[u] = a.owner[k];
      page[u] = a.taken[k];
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      const long long at = t0 + u * rows_a_pass + i;
      const HeadPlan h = a.plan[owner[u]];
      const int k = (int)((at < total ? at : t0) >> p.page_shift), in_page = (int)at & (P - 1);
      const long long t = ((long long)(h.stay + k - h.fresh_at) << p.page_shift) + in_page;
      on[u] = at < total && t < h.n;
      int r = (int)t;
      if (h.list >= 0 && on[u]) r = p.kept_idx[(long long)(owner[u] / G) * p.kept_capacity + h.list + t];
      on[u] = on[u] && r >= 0 && r < h.old;
      src[u] = on[u] ? ((long long)tables[(long long)h.from * p.max_blocks + (r >> p.page_shift)] << p.page_shift) + (r & (P - 1)) : 0;
      dst[u] = ((long long)page[u] << p.page_shift) + in_page;
    }
    u32x4 kx[ROWS], vx[ROWS];
    int px[ROWS];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {                  // a row that is not there: row 0 of the pool, which is
      kx[u] = k_in[src[u] * per_row + x];
      vx[u] = v_in[src[u] * per_row + x];
      px[u] = p.pos != nullptr && x == 0 ? p.pos[src[u]] : 0;
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      if (on[u]) {
        k_out[dst[u] * per_row + x] = kx[u];
        v_out[dst[u] * per_row + x] = vx[u];
        if (p.pos != nullptr && x == 0) p.pos[dst[u]] = px[u];
      }
    }
  }
  // heads, a wavefront each: tables and counts
  for (int h = wave0; h < a.heads; h += waves) {
    const HeadPlan y = a.plan[h];
    const long long row = (long long)h * p.max_blocks, from = (long long)y.from * p.max_blocks;
    const int nb = blocks_of(p, y.n);
    for (int j = (table_apart || y.from != h ? 0 : y.stay) + lane; j < nb; j += 64)
      p.table_out[row + j] = j >= y.stay ? a.taken[y.fresh_at + j - y.stay] : tables[from + j];
    if (lane == 0) {
      p.st.head_rows_out[h] = y.n;
      if (h % G == 0) p.st.seq_pos_out[h / G] = a.seq_pos[h / G];
    }
  }
  if (back == 0) return;                                       // uniform: the same for all
  // pages given back
  for (int h = wave0; h < a.heads; h += waves) {
    int* to = p.free_out + left + s_before[a.one != 0 ? 0 : h / (kChangeWaves * a.per)] + a.plan[h].back_at;
    for_each_gone(a, h, tables + (long long)h * p.max_blocks, [to](int page, int n) { to[n] = page; });
  }
}

}  // namespace

size_t page_change_bytes(int32_t batch, int32_t n_kv_heads, int32_t max_blocks, int64_t n_pages) {
  return change_layout(batch, n_kv_heads, max_blocks, n_pages).bytes;
}

int32_t launch_page_change(const PageChangeArgs& p, void* ws, hipStream_t s) {
  ChangeArgs a;
  a.p = p;
  a.heads = p.batch * p.heads;
  a.one = a.heads <= kOneHeads && (long long)a.heads * p.max_blocks <= kOneEntries ? 1 : 0;
  a.per = (a.heads + kChangeWaves * kMostGroups - 1) / (kChangeWaves * kMostGroups);
  const int groups = a.one != 0 ? 1 : (a.heads + kChangeWaves * a.per - 1) / (kChangeWaves * a.per);
  const ChangeLayout l = change_layout(p.batch, p.heads, p.max_blocks, p.n_pages);
  char* w = static_cast<char*>(ws);
  a.head = reinterpret_cast<ChangeHeader*>(w);
  a.fresh_total = reinterpret_cast<int*>(w + l.off_fresh);
  a.back_total = reinterpret_cast<int*>(w + l.off_back);
  a.seq_pos = reinterpret_cast<int*>(w + l.off_pos);
  a.old_rows = reinterpret_cast<int*>(w + l.off_rows);
  a.plan = reinterpret_cast<HeadPlan*>(w + l.off_plan);
  a.alive = reinterpret_cast<unsigned int*>(w + l.off_alive);
  a.first = reinterpret_cast<unsigned int*>(w + l.off_first);
  a.taken = reinterpret_cast<int*>(w + l.off_taken);
  a.owner = reinterpret_cast<int*>(w + l.off_owner);
  a.old_table = p.table_out == p.st.block_table ? reinterpret_cast<int*>(w + l.off_table) : nullptr;
  {
    ProfScope ps(KID_PAGE_MARK, s);
    if (a.one != 0) {
      hipLaunchKernelGGL(change_one_kernel, dim3(1), dim3(kOneThreads), 0, s, a);
    } else {
      const long long wgs = (p.n_pages + 1023) / 1024;
      hipLaunchKernelGGL(change_begin_kernel, dim3((unsigned)(wgs < 2048 ? wgs : 2048)), dim3(256), 0, s, a);
      hipLaunchKernelGGL(change_mark_kernel, dim3((unsigned)groups), dim3(kChangeThreads), 0, s, a);
      hipLaunchKernelGGL(change_count_kernel, dim3((unsigned)groups), dim3(kChangeThreads), 0, s, a);
    }
  }
  int32_t st = launch_status();
  if (st != LAVA_OK) return st;
  // as many workgroups as there can be work for, up to two rounds of what the device holds: of a fork a head copies less than a page.
  // Rows from anywhere, and few rows, are copied two at a time (32 caches evicted 21.3 -> 20.0 us, eight beams' pages 9.0 -> 8.1), long
  // runs four (64 samples of 8 prompts 17.3 -> 16.0).
  const long long rows = (long long)a.heads * ((p.head_counts != nullptr ? p.max_blocks : 1LL) << p.page_shift);
  const bool four = p.head_counts == nullptr && rows > 8192;
  const long long pass = (long long)kApplyThreads / (p.row_bytes >> 4) * (four ? 4 : 2);
  long long wgs = (rows + pass - 1) / pass;
  if (wgs < (a.heads + kApplyWaves - 1) / kApplyWaves) wgs = (a.heads + kApplyWaves - 1) / kApplyWaves;
  if (wgs > kMostApply) wgs = kMostApply;
  ProfScope ps(KID_PAGE_APPLY, s);
  if (four) hipLaunchKernelGGL(change_apply_kernel<4>, dim3((unsigned)wgs), dim3(kApplyThreads), 0, s, a, groups);
  else hipLaunchKernelGGL(change_apply_kernel<2>, dim3((unsigned)wgs), dim3(kApplyThreads), 0, s, a, groups);
  return launch_status();
}

}  // namespace lava
