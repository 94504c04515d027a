// C ABI of the paged cache: argument checks on the host, then kernel launches on the caller's stream.
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

// What the kernels read of a rotary descriptor.
int32_t check_rotary(const lava_rotary_desc* r, int32_t head_dim) {
  if (r == nullptr) return LAVA_ERR_INVALID_ARG;
  if (r->rotary_dim < 2 || (r->interleaved != 0 && r->interleaved != 1)) return LAVA_ERR_INVALID_ARG;
  if (!(r->magnitude >= 0.0f) || r->magnitude > 1e30f) return LAVA_ERR_INVALID_ARG;
  if (r->rotary_dim % 2 != 0 || r->rotary_dim > head_dim) return LAVA_ERR_SHAPE;
  return LAVA_OK;
}

float magnitude_of(const lava_rotary_desc& r) { return r.magnitude > 0.0f ? r.magnitude : 1.0f; }

// The stride of `count` rows; one row has none, whatever the caller names.
bool take_stride(int64_t* stride, int64_t count, int64_t elem) {
  if (count <= 1) *stride = 0;
  return *stride >= 0 && *stride < (int64_t)1 << 48 && *stride * elem % 16 == 0;
}

}  // namespace
}  // namespace lava

using namespace lava;

extern "C" {

size_t lava_page_tables_workspace_bytes(int32_t batch, int32_t n_kv_heads) {
  if (batch < 1 || batch > 65535 || n_kv_heads < 1 || n_kv_heads > 64) return 0;
  if ((int64_t)batch * n_kv_heads > (int64_t)1 << 20) return 0;
  return page_tables_bytes(batch, n_kv_heads);
}

int32_t lava_page_tables(const lava_page_pool* pool, int32_t batch, int32_t n_kv_heads,
                         const lava_page_state* state, const int32_t* n_new, const int32_t* head_counts,
                         const int32_t* release, int64_t max_tokens, int64_t* slots, int32_t* positions,
                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int32_t st = check_pool_sizes(pool, true);
  if (st != LAVA_OK) return st;
  if (batch < 1 || n_kv_heads < 1 || state == nullptr || max_tokens < 0) return LAVA_ERR_INVALID_ARG;
  const lava_page_state& S = *state;
  if (S.block_table == nullptr || S.head_rows == nullptr || S.seq_pos == nullptr || S.free_pages == nullptr ||
      S.n_free == nullptr || S.head_rows_out == nullptr || S.seq_pos_out == nullptr || S.n_free_out == nullptr)
    return LAVA_ERR_INVALID_ARG;
  if (head_counts != nullptr && (slots != nullptr || positions != nullptr || max_tokens != 0)) return LAVA_ERR_INVALID_ARG;
  if (max_tokens == 0 && (slots != nullptr || positions != nullptr)) return LAVA_ERR_INVALID_ARG;
  if (batch > 65535 || n_kv_heads > 64 || (int64_t)batch * n_kv_heads > (int64_t)1 << 20 ||
      max_tokens >= ((int64_t)1 << 31) / n_kv_heads)
    return LAVA_ERR_SHAPE;
  if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) % kAlign) != 0 ||
      workspace_bytes < page_tables_bytes(batch, n_kv_heads))
    return LAVA_ERR_WORKSPACE;
  PageTablesArgs a;
  a.st = S;
  a.n_new = n_new;
  a.head_counts = head_counts;
  a.release = release;
  a.n_pages = pool->n_pages;
  a.max_tokens = slots != nullptr || positions != nullptr ? max_tokens : 0;
  a.slots = reinterpret_cast<long long*>(slots);
  a.positions = positions;
  a.batch = batch;
  a.heads = n_kv_heads;
  a.max_blocks = pool->max_blocks;
  a.page_shift = page_shift_of(pool->page_rows);
  a.ws = workspace;
  discard_stale_error();
  return launch_page_tables(a, static_cast<hipStream_t>(hip_stream));
}

int32_t lava_compact_paged(const lava_layer_desc* desc, int32_t n_problems,
                           const lava_paged_compact_problem* problems, const lava_page_pool* pool,
                           void* hip_stream) {
  int32_t st = check_desc(desc);
  if (st == LAVA_OK) st = check_pool(pool, true);
  if (st != LAVA_OK) return st;
  if (n_problems < 1 || problems == nullptr) return LAVA_ERR_INVALID_ARG;
  for (int i = 0; i < n_problems; ++i) {
    const lava_paged_compact_problem& p = problems[i];
    if (p.k_src == nullptr || p.v_src == nullptr || p.head_offsets == nullptr || (p.kept_idx == nullptr && p.capacity > 0) ||
        p.block_table == nullptr || p.src_rows < 1 || p.capacity < 0 || !aligned16(p.k_src) || !aligned16(p.v_src) ||
        p.table_blocks < 0)
      return LAVA_ERR_INVALID_ARG;
    if (p.table_blocks != 0 && p.table_blocks != pool->max_blocks) return LAVA_ERR_SHAPE;
    if (p.capacity > (p.src_offsets ? p.src_rows : (int64_t)desc->n_kv_heads * p.src_rows)) return LAVA_ERR_BUDGET;
  }
  discard_stale_error();
  return launch_compact_paged(*desc, n_problems, problems, *pool, static_cast<hipStream_t>(hip_stream));
}

int32_t lava_rotary_turns(const lava_rotary_desc* rot, uint64_t* turns) {
  const int32_t st = check_rotary(rot, 128);
  if (st != LAVA_OK) return st;
  const double factor = rot->factor != 0.0 ? rot->factor : 1.0;
  if (turns == nullptr || !(rot->base > 1.0) || !(rot->base <= 1e300) || !(factor >= 1.0) || !(factor <= 1e300) ||
      rot->original_context < 0)
    return LAVA_ERR_INVALID_ARG;
  if (rot->original_context > 0 && !(rot->low_turns >= 0.0 && rot->high_turns > rot->low_turns && rot->high_turns <= 1e300))
    return LAVA_ERR_INVALID_ARG;
  const long double two_pi = 6.283185307179586476925286766559L;
  for (int i = 0; i < rot->rotary_dim / 2; ++i) {
    const long double f = powl((long double)rot->base, -2.0L * i / rot->rotary_dim);   // <= 1 radian a token
    long double g = f / factor;
    if (rot->original_context > 0) {
      const long double r = rot->original_context * f / two_pi;
      long double c = (r - rot->low_turns) / ((long double)rot->high_turns - rot->low_turns);
      c = c < 0.0L ? 0.0L : c > 1.0L ? 1.0L : c;
      g = c * f + (1.0L - c) * f / factor;
    }
    turns[i] = (uint64_t)(g / two_pi * 18446744073709551616.0L + 0.5L);
  }
  return LAVA_OK;
}

int32_t lava_rotary(const lava_rotary_desc* rot, const uint64_t* turns, int32_t dtype, int32_t head_dim,
                    int64_t n_tokens, int32_t n_heads, const int32_t* positions, const void* x,
                    int64_t x_token_stride, int64_t x_head_stride, void* out, int64_t out_token_stride,
                    int64_t out_head_stride, int32_t transpose, void* hip_stream) {
  if (dtype != LAVA_F32 && dtype != LAVA_BF16) return LAVA_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return LAVA_ERR_SHAPE;
  const int32_t st = check_rotary(rot, head_dim);
  if (st != LAVA_OK) return st;
  if (n_tokens < 0 || n_heads < 1) return LAVA_ERR_INVALID_ARG;
  if (n_tokens == 0) return LAVA_OK;                                 // empty buffers may have no address
  if (turns == nullptr || positions == nullptr || x == nullptr || out == nullptr || !aligned16(x) || !aligned16(out))
    return LAVA_ERR_INVALID_ARG;
  const int64_t elem = dtype == LAVA_BF16 ? 2 : 4;
  if (!take_stride(&x_token_stride, n_tokens, elem) || !take_stride(&x_head_stride, n_heads, elem) ||
      !take_stride(&out_token_stride, n_tokens, elem) || !take_stride(&out_head_stride, n_heads, elem))
    return LAVA_ERR_INVALID_ARG;
  if (out == x && (x_token_stride != out_token_stride || x_head_stride != out_head_stride)) return LAVA_ERR_INVALID_ARG;
  if (n_tokens >= (int64_t)1 << 31 || n_heads > 1024) return LAVA_ERR_SHAPE;
  // rows of the output may not share memory: the heads lie inside a token's stride or the tokens inside a head's
  const auto apart = [head_dim](int64_t inner, int64_t n_inner, int64_t outer, int64_t n_outer) {
    if (n_inner > 1 && inner < head_dim) return false;
    return n_outer <= 1 || (outer >= head_dim && (n_inner <= 1 || (outer - head_dim) / (n_inner - 1) >= inner));
  };
  if (!apart(out_head_stride, n_heads, out_token_stride, n_tokens) && !apart(out_token_stride, n_tokens, out_head_stride, n_heads))
    return LAVA_ERR_INVALID_ARG;
  RotaryArgs a = {};
  a.turns = reinterpret_cast<const unsigned long long*>(turns);
  a.positions = positions;
  a.n_tokens = n_tokens;
  a.x = static_cast<const char*>(x);
  a.out = static_cast<char*>(out);
  a.x_token = x_token_stride * elem;
  a.x_head = x_head_stride * elem;
  a.out_token = out_token_stride * elem;
  a.out_head = out_head_stride * elem;
  a.hq = n_heads;
  a.rot = rot->rotary_dim;
  a.interleaved = rot->interleaved;
  a.cos_mul = magnitude_of(*rot);
  a.sin_mul = transpose != 0 ? -a.cos_mul : a.cos_mul;
  discard_stale_error();
  return launch_rotary(a, dtype, head_dim, static_cast<hipStream_t>(hip_stream));
}

int32_t lava_rotary_append(const lava_layer_desc* desc, const lava_rotary_desc* rot, const uint64_t* turns,
                           int64_t n_tokens, const int32_t* positions, const void* q, int64_t q_token_stride,
                           const void* k, int64_t k_token_stride, const void* v, int64_t v_token_stride,
                           void* q_out, const lava_page_pool* pool, const int64_t* slots, void* hip_stream) {
  int32_t st = check_desc(desc);
  if (st == LAVA_OK) st = check_rotary(rot, desc->head_dim);
  if (st == LAVA_OK) st = check_pool(pool, false);
  if (st != LAVA_OK) return st;
  if (n_tokens < 0) return LAVA_ERR_INVALID_ARG;
  if (n_tokens == 0) return LAVA_OK;                                 // empty buffers may have no address
  if (turns == nullptr || positions == nullptr || k == nullptr || v == nullptr || slots == nullptr || (q == nullptr) != (q_out == nullptr))
    return LAVA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out)) return LAVA_ERR_INVALID_ARG;
  const int64_t elem = desc->dtype == LAVA_BF16 ? 2 : 4;
  const int64_t q_row = (int64_t)desc->n_q_heads * desc->head_dim;
  if (!take_stride(&q_token_stride, n_tokens, elem) || !take_stride(&k_token_stride, n_tokens, elem) ||
      !take_stride(&v_token_stride, n_tokens, elem))
    return LAVA_ERR_INVALID_ARG;
  if (q != nullptr && q == q_out && n_tokens > 1 && q_token_stride != q_row) return LAVA_ERR_INVALID_ARG;
  if (n_tokens >= ((int64_t)1 << 31) / desc->n_kv_heads) return LAVA_ERR_SHAPE;
  RotaryArgs a = {};
  a.turns = reinterpret_cast<const unsigned long long*>(turns);
  a.positions = positions;
  a.n_tokens = n_tokens;
  a.x = static_cast<const char*>(q);
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.out = static_cast<char*>(q_out);
  a.x_token = q_token_stride * elem;
  a.k_token = k_token_stride * elem;
  a.v_token = v_token_stride * elem;
  a.x_head = a.out_head = desc->head_dim * elem;
  a.out_token = q_row * elem;
  a.k_pages = static_cast<char*>(pool->k);
  a.v_pages = static_cast<char*>(pool->v);
  a.pos_pages = pool->pos;
  a.slots = reinterpret_cast<const long long*>(slots);
  a.pool_rows = pool->n_pages * pool->page_rows;
  a.hq = q != nullptr ? desc->n_q_heads : 0;
  a.hkv = desc->n_kv_heads;
  a.rot = rot->rotary_dim;
  a.interleaved = rot->interleaved;
  a.cos_mul = a.sin_mul = magnitude_of(*rot);
  discard_stale_error();
  return launch_rotary(a, desc->dtype, desc->head_dim, static_cast<hipStream_t>(hip_stream));
}

size_t lava_paged_decode_workspace_bytes(const lava_layer_desc* desc) {
  lava_layer_desc d;
  if (check_desc_decode(desc, &d) != LAVA_OK) return 0;
  return paged_decode_bytes(d);
}

int32_t lava_paged_decode(const lava_layer_desc* desc, int32_t batch, const void* q, const lava_page_pool* pool,
                          const int32_t* block_table, const int32_t* head_rows, const lava_decode_options* options,
                          const int32_t* q_pos, float* out, float* lse, void* workspace, size_t workspace_bytes,
                          void* hip_stream) {
  lava_layer_desc d;
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
  if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) % kAlign) != 0 ||
      workspace_bytes < paged_decode_bytes(d))
    return LAVA_ERR_WORKSPACE;
  PagedDecodeArgs a;
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
  discard_stale_error();
  return launch_paged_decode(d, a, workspace, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
