// Sequences that become copies of others, lose rows or end, over pages that sequences share.
//
// A new head takes rows of an old one: all of them (fork) or the ascending list r_0 < r_1 < .. that a selection keeps (compact).  With
// `same` the number of leading t with r_t = t, the first floor(same / P) blocks are blocks of the old table, and so is the
// last one where the head keeps all rows of a last page that was not full and is the copy that goes on with it.  The blocks
// behind them go to fresh pages, whose rows are copied.  A page is free afterwards if no new table names it.
//
// Who holds a page is found out by marking, one word a page: a new table's leading blocks store 0, an old table's blocks that
// do not stay take the minimum with 1 + the head's number.  What is left at 1 + h was first named by head h and is in no new
// table: head h gives it back, so that the stack's order does not depend on the order of the marks.
//
// Four launches, since each needs all of what the one before found: clear the marks; mark, and sum the fresh pages over the heads
// (a wavefront a head, partial sums by workgroup); count what goes back, and take the fresh pages off the stack; write tables,
// counts, stack, and copy rows.  What the last launch reads of buffers that it also writes was set aside before.
//
// Bound by the chain of launches for a beam step (one layer of eight beams), by HBM for many rows.
#include "common.h"
#include "decode_parts.h"
#include "tile_ring.h"

namespace lava {

namespace {

constexpr int kChangeWaves = 16, kChangeThreads = kChangeWaves * 64;
constexpr int kMostGroups = 1024;             // workgroups of a launch that sums over heads
constexpr unsigned int kNoHolder = 0xffffffffu;

struct ChangeHeader {
  int error;                                  // LAVA_PAGES_* bits
  int n_free;
};

struct ChangeArgs {
  PageChangeArgs p;
  ChangeHeader* head;
  int *fresh_total, *back_total;              // [kMostGroups] of a workgroup's heads
  int* keeper;                                // [batch] non-zero: the sequence goes on with its source's last pages
  int *seq_src, *seq_pos;                     // [batch] source (-1: none), position after the call
  int *old_rows, *n_new, *stay, *fresh_at, *back_at;     // [heads] rows before, rows and leading blocks after; sums of the heads of the workgroup before
  long long* list_at;                         // [heads] first entry of the head's list in the sequence's, -1: the head keeps all rows
  unsigned int* mark;                         // [n_pages]
  int* taken;                                 // [n_pages] fresh pages in order
  int* old_table;                             // [heads][max_blocks] a copy, if the tables change in place
  int heads, per;                             // heads in all, heads a wavefront
};

struct ChangeLayout {
  size_t off_fresh, off_back, off_keeper, off_src, off_pos, off_heads, off_list, off_mark, off_taken, off_table, bytes;
};
ChangeLayout change_layout(int batch, int n_kv_heads, int max_blocks, long long n_pages) {
  ChangeLayout l;
  const size_t heads = (size_t)batch * n_kv_heads;
  l.off_fresh = align_up(sizeof(ChangeHeader));
  l.off_back = l.off_fresh + align_up(kMostGroups * 4);
  l.off_keeper = l.off_back + align_up(kMostGroups * 4);
  l.off_src = l.off_keeper + align_up((size_t)batch * 4);
  l.off_pos = l.off_src + align_up((size_t)batch * 4);
  l.off_heads = l.off_pos + align_up((size_t)batch * 4);
  l.off_list = l.off_heads + 5 * align_up(heads * 4);
  l.off_mark = l.off_list + align_up(heads * 8);
  l.off_taken = l.off_mark + align_up((size_t)n_pages * 4);
  l.off_table = l.off_taken + align_up((size_t)n_pages * 4);
  l.bytes = l.off_table + align_up(heads * max_blocks * 4);
  return l;
}

// ---------------------------------------------------------------- 1: clear; who goes on with the last page of a sequence
__global__ void __launch_bounds__(256) change_begin_kernel(const ChangeArgs a) {
  const int lane = threadIdx.x & 63;
  const long long step = (long long)gridDim.x * 256;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.head->error = 0;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < a.p.n_pages; i += step) a.mark[i] = kNoHolder;
  if (a.p.source == nullptr) return;
  const int waves = (int)(step / 64);
  for (int b = blockIdx.x * 4 + (threadIdx.x >> 6); b < a.p.batch; b += waves) {     // a wavefront a sequence
    const int s = a.p.source[b];
    bool first = s >= 0 && s < a.p.batch;
    if (first && s != b) {
      first = a.p.source[s] != s;
      for (int c0 = 0; first && c0 < b; c0 += 64) first = __ballot(c0 + lane < b && a.p.source[c0 + lane] == s) == 0ull;
    }
    if (lane == 0) a.keeper[b] = first ? 1 : 0;
  }
}

// Exclusive sums over a workgroup's heads of what its wavefronts found (lane 0 wrote the sums inside the wavefront to out[h]).
__device__ __forceinline__ void sums_of_group(const ChangeArgs& a, int* s_wave, int mine, int* out, int* totals, int h0, int h1) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane == 0) s_wave[wave] = mine;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kChangeWaves; ++w) {
    before += w < wave ? s_wave[w] : 0;
    all += s_wave[w];
  }
  if (lane == 0 && before != 0)
    for (int h = h0; h < h1; ++h) out[h] += before;
  if (threadIdx.x == 0) totals[blockIdx.x] = all;
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

// ---------------------------------------------------------------- 2: what every head keeps; marks; sums of the fresh pages
__global__ void __launch_bounds__(kChangeThreads) change_mark_kernel(const ChangeArgs a) {
  __shared__ int s_wave[kChangeWaves];
  const PageChangeArgs& p = a.p;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, G = p.heads, P = 1 << p.page_shift;
  const int h0 = (blockIdx.x * kChangeWaves + wave) * a.per, h1 = h0 + a.per < a.heads ? h0 + a.per : a.heads;
  const long long most = (long long)p.max_blocks << p.page_shift;
  int error = 0, sum = 0;
  for (int h = h0; h < h1; ++h) {
    const int b = h / G, g = h - b * G;
    int rows = p.st.head_rows[h];
    if (rows < 0 || rows > most) error = LAVA_PAGES_INVALID, rows = 0;
    const int nb_old = (int)(((long long)rows + P - 1) >> p.page_shift);
    int s = p.source != nullptr ? p.source[b] : b;
    if (s < -1 || s >= p.batch) error = LAVA_PAGES_INVALID, s = -1;
    int old = s >= 0 ? p.st.head_rows[s * G + g] : 0;
    if (old < 0 || old > most) old = 0;                        // that head's wavefront reports it
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
        error = LAVA_PAGES_INVALID;
        n = same = 0;
      } else {
        n = (int)lane_value((unsigned int)count, g);
        begin = before;
        same = leading_same(p.kept_idx + (long long)b * p.kept_capacity + begin, n);
      }
    }
    int stay = same >> p.page_shift;
    if ((n & (P - 1)) != 0 && same >= n && (old & (P - 1)) != 0 && n >> p.page_shift == old >> p.page_shift &&
        (p.source == nullptr || a.keeper[b] != 0))
      ++stay;
    const int* mine = p.st.block_table + (long long)h * p.max_blocks;
    if (s >= 0) {
      const int* from = p.st.block_table + ((long long)s * G + g) * p.max_blocks;
      for (int j = lane; j < stay; j += 64) {
        const int page = from[j];
        if (page < 0 || page >= p.n_pages) error = LAVA_PAGES_INVALID;
        else __hip_atomic_store(&a.mark[page], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
    const int kept = s == b ? stay : 0;                        // leading blocks that this head marks itself
    for (int j = lane; j < nb_old; j += 64) {
      const int page = mine[j];
      if (a.old_table != nullptr) a.old_table[(long long)h * p.max_blocks + j] = page;
      if (j < kept) continue;
      if (page < 0 || page >= p.n_pages) error = LAVA_PAGES_INVALID;
      else __hip_atomic_fetch_min(&a.mark[page], 1u + (unsigned int)h, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (lane == 0) {
      a.old_rows[h] = rows;
      a.n_new[h] = n;
      a.stay[h] = stay;
      a.list_at[h] = begin;
      a.fresh_at[h] = sum;
      if (g == 0) {
        a.seq_src[b] = s;
        a.seq_pos[b] = s >= 0 ? p.st.seq_pos[s] : 0;
      }
    }
    sum += (int)(((long long)n + P - 1) >> p.page_shift) - stay;
  }
  if (error != 0) atomicOr(&a.head->error, error);
  sums_of_group(a, s_wave, sum, a.fresh_at, a.fresh_total, h0, h1);
}

// Sums of the workgroups' totals in front of workgroup `group` (x) and of all (y), in every thread of a workgroup.
template <int THREADS>
__device__ __forceinline__ int2 sum_totals(const int* totals, int groups, int group, int* s_sum) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int before = 0, all = 0;
  for (int i = threadIdx.x; i < groups; i += THREADS) {
    const int x = totals[i];
    before += i < group ? x : 0;
    all += x;
  }
  before = (int)lane_value(wave_incl((unsigned int)before), 63);
  all = (int)lane_value(wave_incl((unsigned int)all), 63);
  if (lane == 0) {
    s_sum[2 * wave] = before;
    s_sum[2 * wave + 1] = all;
  }
  __syncthreads();
  int2 r = make_int2(0, 0);
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    r.x += s_sum[2 * w];
    r.y += s_sum[2 * w + 1];
  }
  __syncthreads();
  return r;
}

// ---------------------------------------------------------------- 3: sums of what goes back; the fresh pages
__global__ void __launch_bounds__(kChangeThreads) change_count_kernel(const ChangeArgs a) {
  __shared__ int s_wave[kChangeWaves], s_sum[2 * kChangeWaves];
  const PageChangeArgs& p = a.p;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, G = p.heads;
  const int h0 = (blockIdx.x * kChangeWaves + wave) * a.per, h1 = h0 + a.per < a.heads ? h0 + a.per : a.heads;
  int sum = 0;
  for (int h = h0; h < h1; ++h) {
    const int b = h / G, nb_old = (int)(((long long)a.old_rows[h] + (1 << p.page_shift) - 1) >> p.page_shift), first = a.seq_src[b] == b ? a.stay[h] : 0;
    const int* table = p.st.block_table + (long long)h * p.max_blocks;
    int n = 0;
    for (int j0 = first; j0 < nb_old; j0 += 64) {
      const int j = j0 + lane, page = j < nb_old ? table[j] : -1;
      n += __popcll(__ballot(page >= 0 && page < p.n_pages && a.mark[page] == 1u + (unsigned int)h));
    }
    if (lane == 0) a.back_at[h] = sum;
    sum += n;
  }
  sums_of_group(a, s_wave, sum, a.back_at, a.back_total, h0, h1);
  const int fresh = sum_totals<kChangeThreads>(a.fresh_total, gridDim.x, 0, s_sum).y, n_free = p.st.n_free[0];
  if (blockIdx.x == 0 && threadIdx.x == 0) a.head->n_free = n_free;
  if (n_free < 0 || n_free > p.n_pages || fresh > n_free) return;
  for (int k = blockIdx.x * kChangeThreads + threadIdx.x; k < fresh; k += gridDim.x * kChangeThreads) {
    const int page = p.st.free_pages[n_free - 1 - k];
    if (page < 0 || page >= p.n_pages) atomicOr(&a.head->error, LAVA_PAGES_INVALID);
    a.taken[k] = page;
  }
}

// ---------------------------------------------------------------- 4: tables, counts, stack; rows
constexpr int kApplyThreads = 256, kRowsInFlight = 4;
__global__ void __launch_bounds__(kApplyThreads) change_apply_kernel(const ChangeArgs a, int groups, int chunks) {
  __shared__ int s_sum[2 * kApplyThreads / 64];
  const PageChangeArgs& p = a.p;
  const int h = blockIdx.x / chunks, chunk = blockIdx.x - h * chunks, lane = threadIdx.x & 63;
  const int G = p.heads, b = h / G, g = h - b * G, P = 1 << p.page_shift;
  const int group = h / (kChangeWaves * a.per);
  const int2 fresh = sum_totals<kApplyThreads>(a.fresh_total, groups, group, s_sum);
  const int2 back = sum_totals<kApplyThreads>(a.back_total, groups, group, s_sum);
  const int n_free = a.head->n_free;
  int error = a.head->error;
  if (n_free < 0 || n_free > p.n_pages) error |= LAVA_PAGES_INVALID;
  if (error == 0 && fresh.y > n_free) error = LAVA_PAGES_EXHAUSTED;
  if (error == 0 && (long long)n_free - fresh.y + back.y > p.n_pages) error = LAVA_PAGES_INVALID;
  const int left = error != 0 ? (n_free < 0 ? 0 : n_free > p.n_pages ? (int)p.n_pages : n_free) : n_free - fresh.y;
  const bool table_apart = p.table_out != p.st.block_table;
  int* table_out = p.table_out + (long long)h * p.max_blocks;
  if (p.free_out != p.st.free_pages)
    for (int i = blockIdx.x * kApplyThreads + threadIdx.x; i < left; i += gridDim.x * kApplyThreads) p.free_out[i] = p.st.free_pages[i];
  const int* tables = table_apart ? p.st.block_table : a.old_table;
  const int nb_old = (int)(((long long)a.old_rows[h] + P - 1) >> p.page_shift);
  if (error != 0) {                                            // nothing changes
    if (chunk != 0) return;
    if (table_apart)
      for (int j = threadIdx.x; j < nb_old; j += kApplyThreads) table_out[j] = tables[(long long)h * p.max_blocks + j];
    if (threadIdx.x == 0) {
      p.st.head_rows_out[h] = p.st.head_rows[h];
      if (g == 0) p.st.seq_pos_out[b] = p.st.seq_pos[b];
      if (h == 0) {
        p.st.n_free_out[0] = n_free;
        if (p.st.error != nullptr) atomicOr(p.st.error, error);
      }
    }
    return;
  }
  const int s = a.seq_src[b], n = a.n_new[h], stay = a.stay[h], nb = (int)(((long long)n + P - 1) >> p.page_shift);
  const int* from = tables + ((long long)(s < 0 ? 0 : s) * G + g) * p.max_blocks;   // read where the source has blocks
  const int* fresh_pages = a.taken + fresh.x + a.fresh_at[h];
  if (chunk == 0) {
    for (int j = threadIdx.x; j < nb; j += kApplyThreads) {
      if (j >= stay) table_out[j] = fresh_pages[j - stay];
      else if (table_apart || s != b) table_out[j] = from[j];
    }
    if (threadIdx.x == 0) {
      p.st.head_rows_out[h] = n;
      if (g == 0) p.st.seq_pos_out[b] = a.seq_pos[b];
      if (h == 0) p.st.n_free_out[0] = left + back.y;
    }
    if (threadIdx.x < 64) {                                    // the pages that this head gives back, in the order of its blocks
      const int* mine = tables + (long long)h * p.max_blocks;
      int* to = p.free_out + left + back.x + a.back_at[h];
      for (int j0 = s == b ? stay : 0; j0 < nb_old; j0 += 64) {
        const int j = j0 + lane, page = j < nb_old ? mine[j] : -1;
        const bool gone = page >= 0 && a.mark[page] == 1u + (unsigned int)h;
        const unsigned long long all = __ballot(gone);
        if (gone) to[__popcll(all & ((1ull << lane) - 1ull))] = page;
        to += __popcll(all);
      }
    }
  }
  // rows stay * P .. n - 1 of the head, `per_row` threads a row, kRowsInFlight rows of a thread at a time
  const int per_row = p.row_bytes >> 4, rows_a_pass = kApplyThreads / per_row, i = threadIdx.x / per_row, x = threadIdx.x - i * per_row;
  const long long list = a.list_at[h];
  const int* kept = list < 0 ? nullptr : p.kept_idx + (long long)b * p.kept_capacity + list;
  const int old = s < 0 ? 0 : a.old_rows[s * G + g];
  u32x4 *k_out = reinterpret_cast<u32x4*>(p.k), *v_out = reinterpret_cast<u32x4*>(p.v);
  const u32x4 *k_in = k_out, *v_in = v_out;
  const long long pass = (long long)rows_a_pass * kRowsInFlight;
  for (long long t0 = (long long)stay * P + chunk * pass; t0 < n; t0 += chunks * pass) {
    long long src[kRowsInFlight], dst[kRowsInFlight];
    bool on[kRowsInFlight];
#pragma unroll
    for (int u = 0; u < kRowsInFlight; ++u) {
      const long long t = t0 + u * rows_a_pass + i;
      on[u] = t < n;
      int r = (int)t;
      if (kept != nullptr && on[u]) r = kept[t];
      const int block = r >> p.page_shift;
      on[u] = on[u] && r >= 0 && r < old;
      src[u] = on[u] ? ((long long)from[block] << p.page_shift) + (r & (P - 1)) : 0;
      dst[u] = on[u] ? ((long long)fresh_pages[(int)(t >> p.page_shift) - stay] << p.page_shift) + (t & (P - 1)) : 0;
    }
    u32x4 kx[kRowsInFlight], vx[kRowsInFlight];
    int px[kRowsInFlight];
#pragma unroll
    for (int u = 0; u < kRowsInFlight; ++u) {                  // a row that is not there: row 0 of the pool, which is
      kx[u] = k_in[src[u] * per_row + x];
      vx[u] = v_in[src[u] * per_row + x];
      px[u] = p.pos != nullptr && x == 0 ? p.pos[src[u]] : 0;
    }
#pragma unroll
    for (int u = 0; u < kRowsInFlight; ++u) {
      if (on[u]) {
        k_out[dst[u] * per_row + x] = kx[u];
        v_out[dst[u] * per_row + x] = vx[u];
        if (p.pos != nullptr && x == 0) p.pos[dst[u]] = px[u];
      }
    }
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
  a.per = (a.heads + kChangeWaves * kMostGroups - 1) / (kChangeWaves * kMostGroups);
  const int groups = (a.heads + kChangeWaves * a.per - 1) / (kChangeWaves * a.per);
  const ChangeLayout l = change_layout(p.batch, p.heads, p.max_blocks, p.n_pages);
  char* w = static_cast<char*>(ws);
  a.head = reinterpret_cast<ChangeHeader*>(w);
  a.fresh_total = reinterpret_cast<int*>(w + l.off_fresh);
  a.back_total = reinterpret_cast<int*>(w + l.off_back);
  a.keeper = reinterpret_cast<int*>(w + l.off_keeper);
  a.seq_src = reinterpret_cast<int*>(w + l.off_src);
  a.seq_pos = reinterpret_cast<int*>(w + l.off_pos);
  const size_t heads_bytes = align_up((size_t)a.heads * 4);
  int** const per_head[5] = {&a.old_rows, &a.n_new, &a.stay, &a.fresh_at, &a.back_at};
  for (int i = 0; i < 5; ++i) *per_head[i] = reinterpret_cast<int*>(w + l.off_heads + i * heads_bytes);
  a.list_at = reinterpret_cast<long long*>(w + l.off_list);
  a.mark = reinterpret_cast<unsigned int*>(w + l.off_mark);
  a.taken = reinterpret_cast<int*>(w + l.off_taken);
  a.old_table = p.table_out == p.st.block_table ? reinterpret_cast<int*>(w + l.off_table) : nullptr;
  {
    ProfScope ps(KID_PAGE_MARK, s);
    long long wgs = (p.n_pages + 1023) / 1024;
    if (p.source != nullptr && wgs < (p.batch + 3) / 4) wgs = (p.batch + 3) / 4;
    hipLaunchKernelGGL(change_begin_kernel, dim3((unsigned)(wgs < 2048 ? wgs : 2048)), dim3(256), 0, s, a);
    hipLaunchKernelGGL(change_mark_kernel, dim3((unsigned)groups), dim3(kChangeThreads), 0, s, a);
    hipLaunchKernelGGL(change_count_kernel, dim3((unsigned)groups), dim3(kChangeThreads), 0, s, a);
  }
  int32_t st = launch_status();
  if (st != LAVA_OK) return st;
  // Rows that a head can have to copy: of a fork less than a page.
  const long long most = p.head_counts != nullptr ? (long long)p.max_blocks << p.page_shift : ((long long)1 << p.page_shift) - 1;
  const long long pass = (long long)kApplyThreads / (p.row_bytes >> 4) * kRowsInFlight;
  long long chunks = (most + pass - 1) / pass, room = 4096 / a.heads;
  if (chunks > room) chunks = room;
  if (chunks < 1) chunks = 1;
  ProfScope ps(KID_PAGE_APPLY, s);
  hipLaunchKernelGGL(change_apply_kernel, dim3((unsigned)(a.heads * chunks)), dim3(kApplyThreads), 0, s, a, groups, (int)chunks);
  return launch_status();
}

}  // namespace lava
