// C-ABI entry points of what a decoder layer does around its products: argument checks on the host, then one or two launches.
#include "dispatch_rules.h"
#include "moqe_internal.h"

namespace moqe {
namespace {

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int32_t check_norm(const moqe_norm& n, const char* which, const char* who) {
  if (n.kind < MOQE_NORM_NONE || n.kind > MOQE_NORM_LAYER) return set_error(MOQE_E_FORMAT, "%s: %s norm of kind %d", who, which, n.kind);
  if (n.kind != MOQE_NORM_NONE && !(n.eps >= 0.f)) return set_error(MOQE_E_SHAPE, "%s: %s norm has a negative eps", who, which);
  if (n.offset && n.kind != MOQE_NORM_LAYER) return set_error(MOQE_E_FORMAT, "%s: %s norm: only layer norms have an offset", who, which);
  if (!aligned(n.gain, 4) || !aligned(n.offset, 4)) return set_error(MOQE_E_SHAPE, "%s: %s norm: misaligned vector", who, which);
  return MOQE_OK;
}

int32_t check_cache(const moqe_kv_cache* c, const char* who) {
  if (!c) return set_error(MOQE_E_NULL, "%s: cache is NULL", who);
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return set_error(MOQE_E_SHAPE, "%s: head_dim %d is not 64, 128 or 256", who, c->head_dim);
  if (c->block_tokens != 32 && c->block_tokens != 64 && c->block_tokens != 128)
    return set_error(MOQE_E_SHAPE, "%s: block_tokens %d is not 32, 64 or 128", who, c->block_tokens);
  if (c->n_heads < 1 || c->n_heads > 65535 || c->n_blocks < 1)
    return set_error(MOQE_E_SHAPE, "%s: cache of %d blocks and %d heads", who, c->n_blocks, c->n_heads);
  if (!c->k || !c->v || !c->k_scale || !c->v_scale) return set_error(MOQE_E_NULL, "%s: a buffer of the cache is NULL", who);
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))
    return set_error(MOQE_E_SHAPE, "%s: the cache's codes must be 16-byte aligned, its scales 4-byte aligned", who);
  return MOQE_OK;
}

int32_t check_batch(const moqe_kv_batch* b, const moqe_kv_cache& c, const char* who) {
  if (!b) return set_error(MOQE_E_NULL, "%s: batch is NULL", who);
  if (b->S < 0 || b->T < 1 || b->M < 0 || b->table_width < 1)
    return set_error(MOQE_E_SHAPE, "%s: S=%d T=%d M=%d table_width=%d", who, b->S, b->T, b->M, b->table_width);
  if (!b->cu_rows && static_cast<long long>(b->S) * b->T != b->M)
    return set_error(MOQE_E_SHAPE, "%s: M=%d is not S*T=%lld", who, b->M, static_cast<long long>(b->S) * b->T);
  if (static_cast<long long>(b->table_width) * c.block_tokens > (1ll << 30) || b->T > (1 << 24) || static_cast<long long>(b->S) * b->T > (1ll << 30))
    return set_error(MOQE_E_SHAPE, "%s: more than 2^30 tokens a sequence, 2^24 rows a sequence or 2^30 rows", who);
  if (static_cast<long long>(b->S) * b->table_width * c.block_tokens > (1ll << 35))
    return set_error(MOQE_E_SHAPE, "%s: block tables of more than 2^35 tokens in all", who);
  if (b->S > 0 && (!b->block_table || !b->kv_len)) return set_error(MOQE_E_NULL, "%s: block_table or kv_len is NULL", who);
  if (!aligned(b->block_table, 4) || !aligned(b->kv_len, 4) || !aligned(b->cu_rows, 4))
    return set_error(MOQE_E_SHAPE, "%s: misaligned block_table, kv_len or cu_rows", who);
  return MOQE_OK;
}

int32_t check_heads(int32_t n_heads, const moqe_kv_cache& c, const char* who) {
  if (n_heads < 1 || n_heads > 65535 || n_heads % c.n_heads)
    return set_error(MOQE_E_SHAPE, "%s: %d query heads on %d key heads", who, n_heads, c.n_heads);
  return MOQE_OK;
}

int32_t check_rows(const void* p, int64_t stride, long long least, const char* what, const char* who) {
  if (!p) return set_error(MOQE_E_NULL, "%s: %s is NULL", who, what);
  if (!aligned(p, 16) || stride % 8) return set_error(MOQE_E_SHAPE, "%s: %s must be 16-byte aligned with a stride that is a multiple of 8", who, what);
  if (stride < least || stride > (1ll << 32)) return set_error(MOQE_E_SHAPE, "%s: stride %lld of %s, rows have %lld values", who, static_cast<long long>(stride), what, least);
  return MOQE_OK;
}

int32_t check_attention(const moqe_attention* at, const moqe_kv_batch* b, const moqe_kv_cache* c, const char* who) {
  int32_t rc = check_cache(c, who);
  if (!rc) rc = check_batch(b, *c, who);
  if (rc) return rc;
  if (!at) return set_error(MOQE_E_NULL, "%s: attention is NULL", who);
  rc = check_heads(at->n_heads, *c, who);
  if (rc) return rc;
  if (!(at->scale == at->scale) || !(at->cap >= 0.f)) return set_error(MOQE_E_SHAPE, "%s: scale is NaN or cap is negative", who);
  if (!aligned(at->slopes, 4) || !aligned(at->prefix, 4)) return set_error(MOQE_E_SHAPE, "%s: misaligned slopes or prefix", who);
  return MOQE_OK;
}

// `out8`: results in 8 bits are wanted, so that there need not be others.  *empty: there are no rows.
int32_t check_residual_step(const moqe_residual_step* s, bool out8, const char* who, bool* empty) {
  *empty = false;
  if (!s) return set_error(MOQE_E_NULL, "%s: step is NULL", who);
  if (s->M < 0 || s->d < 1 || s->d > 32768) return set_error(MOQE_E_SHAPE, "%s: %d rows of %d features (1 .. 32768)", who, s->M, s->d);
  if ((s->y_type != MOQE_TYPE_F32 && s->y_type != MOQE_TYPE_BF16) || (s->residual_type != MOQE_TYPE_F32 && s->residual_type != MOQE_TYPE_BF16))
    return set_error(MOQE_E_FORMAT, "%s: y_type %d, residual_type %d", who, s->y_type, s->residual_type);
  int32_t rc = check_norm(s->post, "post", who);
  if (!rc) rc = check_norm(s->pre, "pre", who);
  if (rc) return rc;
  if (s->gate_rows < 0) return set_error(MOQE_E_SHAPE, "%s: gate_rows %d", who, s->gate_rows);
  if (s->M == 0) {
    *empty = true;
    return MOQE_OK;
  }
  if (!s->residual) return set_error(MOQE_E_NULL, "%s: residual is NULL", who);
  if (!s->residual_out && !s->out && !out8) return set_error(MOQE_E_NULL, "%s: residual_out and out are both NULL", who);
  if (s->residual_stride < s->d || (s->y && s->y_stride < s->d) || (s->residual_out && s->residual_out_stride < s->d) || (s->out && s->out_stride < s->d))
    return set_error(MOQE_E_SHAPE, "%s: a row stride is smaller than d = %d", who, s->d);
  if (s->residual_out == s->residual && s->residual_out_stride != s->residual_stride)
    return set_error(MOQE_E_SHAPE, "%s: residual_out is residual with another stride", who);
  const size_t ysz = s->y_type == MOQE_TYPE_F32 ? 4 : 2, rsz = s->residual_type == MOQE_TYPE_F32 ? 4 : 2;
  if (!aligned(s->y, ysz) || !aligned(s->residual, rsz) || !aligned(s->residual_out, rsz) || !aligned(s->out, 2) || !aligned(s->gate, 4))
    return set_error(MOQE_E_SHAPE, "%s: a pointer is not aligned to its type", who);
  return MOQE_OK;
}

}  // namespace
}  // namespace moqe

using namespace moqe;

extern "C" {

int32_t moqe_residual_norm(const moqe_residual_step* s, void* stream) {
  bool empty;
  const int32_t rc = check_residual_step(s, false, "moqe_residual_norm", &empty);
  if (rc || empty || dry_run()) return rc;
  return launch_residual_norm(*s, nullptr, static_cast<hipStream_t>(stream));
}

int32_t moqe_residual_norm_f8(const moqe_residual_step* s, const moqe_f8_rows* out8, void* stream) {
  const char* who = "moqe_residual_norm_f8";
  bool empty;
  int32_t rc = check_residual_step(s, true, who, &empty);
  if (rc || empty) return rc;
  rc = check_f8_rows(out8, s->d, "out8", who);
  if (rc || dry_run()) return rc;
  return launch_residual_norm(*s, out8, static_cast<hipStream_t>(stream));
}

size_t moqe_kv_codes_bytes(const moqe_kv_cache* c) {
  if (!c || c->n_blocks < 1 || c->n_heads < 1 || c->block_tokens < 1 || c->head_dim < 1) return 0;
  return size_t(c->n_blocks) * c->n_heads * c->block_tokens * c->head_dim;
}

int32_t moqe_kv_append(const void* qkv, int32_t qkv_type, int64_t qkv_stride, int32_t n_heads, const moqe_rope* rope, const moqe_kv_batch* batch,
                       const moqe_kv_cache* cache, void* q_out, int64_t q_stride, void* stream) {
  const char* who = "moqe_kv_append";
  int32_t rc = check_cache(cache, who);
  if (!rc) rc = check_batch(batch, *cache, who);
  if (!rc) rc = check_heads(n_heads, *cache, who);
  if (rc) return rc;
  if (qkv_type != MOQE_TYPE_F32 && qkv_type != MOQE_TYPE_BF16) return set_error(MOQE_E_FORMAT, "%s: qkv_type %d", who, qkv_type);
  if (!rope) return set_error(MOQE_E_NULL, "%s: rope is NULL", who);
  if (rope->rot_dim < 0 || rope->rot_dim % 16 || rope->rot_dim > cache->head_dim)
    return set_error(MOQE_E_SHAPE, "%s: rot_dim %d is not a multiple of 16 up to head_dim %d", who, rope->rot_dim, cache->head_dim);
  if (rope->rot_dim > 0 && !rope->inv_freq) return set_error(MOQE_E_NULL, "%s: inv_freq is NULL", who);
  if (!aligned(rope->inv_freq, 8) || !aligned(rope->q_gain, 4) || !aligned(rope->k_gain, 4)) return set_error(MOQE_E_SHAPE, "%s: misaligned rope vectors", who);
  if ((rope->q_gain || rope->k_gain) && !(rope->eps >= 0.f)) return set_error(MOQE_E_SHAPE, "%s: negative eps", who);
  if (batch->S == 0 || batch->M == 0) return MOQE_OK;
  const long long dh = cache->head_dim;
  rc = check_rows(qkv, qkv_stride, (n_heads + 2ll * cache->n_heads) * dh, "qkv", who);
  if (!rc) rc = check_rows(q_out, q_stride, n_heads * dh, "q_out", who);
  if (rc) return rc;
  if (dry_run()) return MOQE_OK;
  return launch_kv_append(qkv, qkv_type == MOQE_TYPE_BF16, qkv_stride, n_heads, *rope, *batch, *cache, q_out, q_stride, static_cast<hipStream_t>(stream));
}

size_t moqe_kv_attention_workspace_bytes(const moqe_attention* at, const moqe_kv_batch* b, const moqe_kv_cache* c) {
  if (check_attention(at, b, c, "moqe_kv_attention_workspace_bytes")) return 0;
  if (b->S == 0 || b->M == 0) return 0;
  return kv_few_rows(b->T, at->n_heads / c->n_heads, c->head_dim) ? kv_attend_few_ws_bytes(*at, *b, *c) : kv_attend_rows_ws_bytes(*at, *b, *c);
}

int32_t moqe_kv_attention(const void* q, int64_t q_stride, const moqe_attention* at, const moqe_kv_batch* b, const moqe_kv_cache* c, void* out,
                          int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "moqe_kv_attention";
  int32_t rc = check_attention(at, b, c, who);
  if (rc) return rc;
  if (b->S == 0 || b->M == 0) return MOQE_OK;
  const long long width = static_cast<long long>(at->n_heads) * c->head_dim;
  rc = check_rows(q, q_stride, width, "q", who);
  if (!rc) rc = check_rows(out, out_stride, width, "out", who);
  if (rc) return rc;
  const size_t need = moqe_kv_attention_workspace_bytes(at, b, c);
  if (need && (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
    return set_error(MOQE_E_WORKSPACE, "%s: workspace needs %zu bytes, 256-byte aligned", who, need);
  if (dry_run()) return MOQE_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (kv_few_rows(b->T, at->n_heads / c->n_heads, c->head_dim)) return launch_kv_attend_few(q, q_stride, *at, *b, *c, out, out_stride, workspace, st);
  return launch_kv_attend_rows(q, q_stride, *at, *b, *c, out, out_stride, workspace, st);
}

}  // extern "C"
