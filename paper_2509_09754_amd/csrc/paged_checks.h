// Argument checks that the entry points of the paged cache and of sequences that share pages have in common.
#pragma once

#include <math.h>

#include "common.h"

namespace lava {
namespace {

int page_shift_of(int32_t page_rows) {
  for (int s = 4; s <= 8; ++s)
    if (page_rows == 1 << s) return s;
  return -1;
}

// The sizes of a pool (what lava_page_tables reads of it).
int32_t check_pool_sizes(const lava_page_pool* p, bool blocks) {
  if (p == nullptr) return LAVA_ERR_INVALID_ARG;
  if (p->n_pages < 1 || p->page_rows < 1 || (blocks && p->max_blocks < 1)) return LAVA_ERR_INVALID_ARG;
  if (p->n_pages >= (int64_t)1 << 31 || page_shift_of(p->page_rows) < 0) return LAVA_ERR_SHAPE;
  if (blocks && (int64_t)p->max_blocks * p->page_rows >= (int64_t)1 << 31) return LAVA_ERR_SHAPE;
  return LAVA_OK;
}

int32_t check_pool(const lava_page_pool* p, bool blocks) {
  const int32_t st = check_pool_sizes(p, blocks);
  if (st != LAVA_OK) return st;
  return p->k == nullptr || p->v == nullptr || !aligned16(p->k) || !aligned16(p->v) ? LAVA_ERR_INVALID_ARG : LAVA_OK;
}

// The arguments of a decode step over pages, all but its workspace: the descriptor for its kernels in *out_desc, theirs in *args.
inline int32_t check_paged_decode(const lava_layer_desc* desc, int32_t batch, const void* q, const lava_page_pool* pool,
                                  const int32_t* block_table, const int32_t* head_rows, const lava_decode_options* options,
                                  const int32_t* q_pos, float* out, float* lse, lava_layer_desc* out_desc, PagedDecodeArgs* args) {
  lava_layer_desc& d = *out_desc;
  int32_t st = check_desc_decode(desc, &d);
  if (st == LAVA_OK) st = check_pool(pool, true);
  if (st != LAVA_OK) return st;
  if (batch < 1 || q == nullptr || block_table == nullptr || head_rows == nullptr || out == nullptr || !aligned16(q))
    return LAVA_ERR_INVALID_ARG;
  lava_decode_options o = {};
  if (options != nullptr) o = *options;
  // the kernel multiplies by the cap's reciprocal, which has to be finite: a logit of zero would give NaN
  if (!(o.softcap >= 0.0f) || o.softcap > 1e30f || (o.softcap > 0.0f && o.softcap < 1e-30f) || o.window < 0) return LAVA_ERR_INVALID_ARG;
  const bool needs_pos = o.window > 0 || o.slopes != nullptr;
  if (needs_pos && (q_pos == nullptr || pool->pos == nullptr || !aligned16(pool->pos))) return LAVA_ERR_INVALID_ARG;
  if (batch > 65535 || (int64_t)batch * d.n_kv_heads > 65536) return LAVA_ERR_SHAPE;
  // the tiles of all heads are counted in 32 bits
  if ((int64_t)batch * d.n_kv_heads > (((int64_t)1 << 35) - 1) / ((int64_t)pool->max_blocks * pool->page_rows)) return LAVA_ERR_SHAPE;
  PagedDecodeArgs& a = *args;
  a.q = static_cast<const char*>(q);
  a.k = static_cast<const char*>(pool->k);
  a.v = static_cast<const char*>(pool->v);
  a.pos = needs_pos ? pool->pos : nullptr;
  a.block_table = block_table;
  a.head_rows = head_rows;
  a.q_pos = q_pos;
  a.slopes = o.slopes;
  a.n_pages = pool->n_pages;
  a.page_shift = page_shift_of(pool->page_rows);
  a.max_blocks = pool->max_blocks;
  a.batch = batch;
  a.H = d.n_q_heads;
  a.H_kv = d.n_kv_heads;
  a.G = d.n_q_heads / d.n_kv_heads;
  a.window = o.window;
  a.scale = d.softmax_scale > 0.0f ? d.softmax_scale : 1.0f / sqrtf((float)d.head_dim);
  a.cap = o.softcap;
  a.out = out;
  a.lse = lse;
  a.sums = nullptr;
  return LAVA_OK;
}

}  // namespace
}  // namespace lava
