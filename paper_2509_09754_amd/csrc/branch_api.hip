// C ABI of sequences that begin alike and share pages: argument checks on the host, then kernel launches on the caller's stream.
#include "common.h"
#include "paged_checks.h"

using namespace lava;

namespace {

bool good_workspace(const void* workspace, size_t bytes, size_t need) {
  return workspace != nullptr && (reinterpret_cast<uintptr_t>(workspace) % kAlign) == 0 && bytes >= need;
}

int32_t check_beams(int32_t batch, int32_t beams, int64_t vocab, int32_t n_out) {
  if (batch < 1 || beams < 1 || vocab < 1 || n_out < 1) return LAVA_ERR_INVALID_ARG;
  if (batch > 65535 || beams > 64 || n_out > 64 || vocab >= (int64_t)1 << 31) return LAVA_ERR_SHAPE;
  if ((int64_t)batch * beams * ((vocab + 8191) / 8192) >= (int64_t)1 << 24) return LAVA_ERR_SHAPE;   // a launch has fewer than 2^32 threads, 256 of them each
  return LAVA_OK;
}

bool change_sizes_fit(int64_t batch, int64_t heads, int64_t blocks, int64_t pages) {
  if (batch < 1 || heads < 1 || blocks < 1 || pages < 1) return false;
  return batch <= 65535 && heads <= 64 && batch * heads <= (int64_t)1 << 20 && blocks < (int64_t)1 << 31 && pages < (int64_t)1 << 31 &&
         batch * heads * blocks < (int64_t)1 << 31;
}

// What forks and compactions share; the caller has filled in what only it has.
int32_t change(const lava_layer_desc* desc, const lava_page_pool* pool, int32_t batch, const lava_page_state* state, PageChangeArgs& a,
               int32_t* block_table_out, int32_t* free_pages_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int32_t st = check_desc(desc);
  if (st == LAVA_OK) st = check_pool(pool, true);
  if (st != LAVA_OK) return st;
  if (batch < 1 || state == nullptr) return LAVA_ERR_INVALID_ARG;
  const lava_page_state& S = *state;
  if (S.block_table == nullptr || S.head_rows == nullptr || S.seq_pos == nullptr || S.free_pages == nullptr ||
      S.n_free == nullptr || S.head_rows_out == nullptr || S.seq_pos_out == nullptr || S.n_free_out == nullptr)
    return LAVA_ERR_INVALID_ARG;
  if (!change_sizes_fit(batch, desc->n_kv_heads, pool->max_blocks, pool->n_pages)) return LAVA_ERR_SHAPE;
  if (!good_workspace(workspace, workspace_bytes, page_change_bytes(batch, desc->n_kv_heads, pool->max_blocks, pool->n_pages)))
    return LAVA_ERR_WORKSPACE;
  a.st = S;
  a.table_out = block_table_out != nullptr ? block_table_out : S.block_table;
  a.free_out = free_pages_out != nullptr ? free_pages_out : S.free_pages;
  a.k = static_cast<char*>(pool->k);
  a.v = static_cast<char*>(pool->v);
  a.pos = pool->pos;
  a.n_pages = pool->n_pages;
  a.batch = batch;
  a.heads = desc->n_kv_heads;
  a.max_blocks = pool->max_blocks;
  a.page_shift = page_shift_of(pool->page_rows);
  a.row_bytes = desc->head_dim * (desc->dtype == LAVA_BF16 ? 2 : 4);
  discard_stale_error();
  return launch_page_change(a, workspace, static_cast<hipStream_t>(hip_stream));
}

}  // namespace

extern "C" {

size_t lava_beam_step_workspace_bytes(int32_t batch, int32_t beams, int64_t vocab, int32_t n_out) {
  return check_beams(batch, beams, vocab, n_out) == LAVA_OK ? beam_step_bytes(batch, beams, vocab, n_out) : 0;
}

int32_t lava_beam_step(int32_t dtype, int32_t batch, int32_t beams, int64_t vocab, const void* logits, int64_t logit_stride,
                       const float* scores, const int32_t* done, int32_t end_token, int32_t pad_token, int32_t n_out,
                       int32_t* parents, int32_t* tokens, float* scores_out, int32_t* done_out, int32_t* sources, int32_t n_tables,
                       void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (dtype != LAVA_F32 && dtype != LAVA_BF16) return LAVA_ERR_INVALID_ARG;
  const int32_t st = check_beams(batch, beams, vocab, n_out);
  if (st != LAVA_OK) return st;
  const int64_t elem = dtype == LAVA_BF16 ? 2 : 4;
  if (logits == nullptr || reinterpret_cast<uintptr_t>(logits) % elem != 0 || scores == nullptr || parents == nullptr ||
      tokens == nullptr || scores_out == nullptr || n_tables < 0 || (sources == nullptr) != (n_tables == 0))
    return LAVA_ERR_INVALID_ARG;
  if (pad_token < 0 || pad_token >= vocab || ((int64_t)batch * beams > 1 && logit_stride < vocab)) return LAVA_ERR_INVALID_ARG;
  if (n_out != beams && (scores_out == scores || (done != nullptr && done_out == done))) return LAVA_ERR_INVALID_ARG;
  if (logit_stride >= (int64_t)1 << 40 || n_tables > 1024) return LAVA_ERR_SHAPE;
  if ((int64_t)n_tables * batch * (beams > n_out ? beams : n_out) >= (int64_t)1 << 31) return LAVA_ERR_SHAPE;
  if (!good_workspace(workspace, workspace_bytes, beam_step_bytes(batch, beams, vocab, n_out))) return LAVA_ERR_WORKSPACE;
  BeamArgs a;
  a.logits = static_cast<const char*>(logits);
  a.vocab = vocab;
  a.stride_bytes = (int64_t)batch * beams > 1 ? logit_stride * elem : 0;
  a.scores = scores;
  a.done = done;
  a.parents = parents;
  a.tokens = tokens;
  a.scores_out = scores_out;
  a.done_out = done_out;
  a.sources = sources;
  a.batch = batch;
  a.beams = beams;
  a.n_out = n_out;
  a.n_tables = n_tables;
  a.end_token = end_token;
  a.pad_token = pad_token;
  discard_stale_error();
  return launch_beam_step(a, dtype, workspace, static_cast<hipStream_t>(hip_stream));
}

size_t lava_page_fork_workspace_bytes(int32_t batch, int32_t n_kv_heads, int32_t max_blocks, int64_t n_pages) {
  return change_sizes_fit(batch, n_kv_heads, max_blocks, n_pages) ? page_change_bytes(batch, n_kv_heads, max_blocks, n_pages) : 0;
}

int32_t lava_page_fork(const lava_layer_desc* desc, const lava_page_pool* pool, int32_t batch, const lava_page_state* state,
                       const int32_t* source, int32_t* block_table_out, int32_t* free_pages_out, void* workspace,
                       size_t workspace_bytes, void* hip_stream) {
  if (source == nullptr) return LAVA_ERR_INVALID_ARG;
  PageChangeArgs a = {};
  a.source = source;
  return change(desc, pool, batch, state, a, block_table_out, free_pages_out, workspace, workspace_bytes, hip_stream);
}

int32_t lava_page_compact(const lava_layer_desc* desc, const lava_page_pool* pool, int32_t batch, const lava_page_state* state,
                          const int32_t* head_counts, const int32_t* kept_idx, int64_t kept_capacity, const int32_t* evict,
                          int32_t* block_table_out, int32_t* free_pages_out, void* workspace, size_t workspace_bytes,
                          void* hip_stream) {
  if (head_counts == nullptr || kept_capacity < 0 || (kept_idx == nullptr && kept_capacity > 0)) return LAVA_ERR_INVALID_ARG;
  if (kept_capacity >= (int64_t)1 << 40) return LAVA_ERR_SHAPE;
  PageChangeArgs a = {};
  a.head_counts = head_counts;
  a.kept_idx = kept_idx;
  a.kept_capacity = kept_capacity;
  a.evict = evict;
  return change(desc, pool, batch, state, a, block_table_out, free_pages_out, workspace, workspace_bytes, hip_stream);
}

size_t lava_shared_decode_workspace_bytes(const lava_layer_desc* desc, int32_t batch, int32_t max_blocks) {
  lava_layer_desc d;
  if (check_desc_decode(desc, &d) != LAVA_OK || batch < 1 || batch > 65535 || max_blocks < 1) return 0;
  if ((int64_t)batch * d.n_kv_heads > 65536 || (int64_t)batch * d.n_kv_heads * max_blocks >= (int64_t)1 << 31) return 0;
  return shared_decode_bytes(d, batch, max_blocks);
}

int32_t lava_shared_decode(const lava_layer_desc* desc, int32_t batch, const void* q, const lava_page_pool* pool,
                           const int32_t* block_table, const int32_t* head_rows, int32_t n_groups, const int32_t* group_start,
                           const lava_decode_options* options, const int32_t* q_pos, float* out, float* lse, void* workspace,
                           size_t workspace_bytes, void* hip_stream) {
  lava_layer_desc d;
  PagedDecodeArgs a;
  const int32_t st = check_paged_decode(desc, batch, q, pool, block_table, head_rows, options, q_pos, out, lse, &d, &a);
  if (st != LAVA_OK) return st;
  if (n_groups < 1 || n_groups > batch || group_start == nullptr) return LAVA_ERR_INVALID_ARG;
  if ((int64_t)batch * d.n_kv_heads * pool->max_blocks >= (int64_t)1 << 31) return LAVA_ERR_SHAPE;
  if (!good_workspace(workspace, workspace_bytes, shared_decode_bytes(d, batch, pool->max_blocks))) return LAVA_ERR_WORKSPACE;
  discard_stale_error();
  return launch_shared_decode(d, a, n_groups, group_start, workspace, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
