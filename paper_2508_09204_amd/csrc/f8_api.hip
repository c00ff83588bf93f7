// C-ABI entry points of rows, matrices and products in 8-bit floating point, and of sampling: argument checks on the host, then the launches.
#include "dispatch_rules.h"
#include "f8_device.h"

namespace moqe {
namespace {

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int32_t check_f8_size(int32_t n, int32_t k, int32_t gated, const char* who) {
  if (n < 1 || k < 1) return set_error(MOQE_E_SHAPE, "%s: matrix of %d x %d", who, n, k);
  if (n > (1 << 30) || k > (1 << 30) || (2ll * n + 32) * (k + 512ll) >= (1ll << 40)) return set_error(MOQE_E_SHAPE, "%s: matrix of %d x %d", who, n, k);
  if (f8_packed(n, k, gated).total >= (size_t(1) << 32)) return set_error(MOQE_E_SHAPE, "%s: packed matrix %d x %d takes 4 GiB or more", who, n, k);
  return MOQE_OK;
}

int32_t check_f8_experts(const moqe_f8_mat* m, int32_t K, const char* who) {
  if (!m) return set_error(MOQE_E_NULL, "%s: experts is NULL", who);
  if (K < 1 || K > MOQE_MAX_EXPERTS) return set_error(MOQE_E_SHAPE, "%s: %d experts, 1 to %d", who, K, MOQE_MAX_EXPERTS);
  const int32_t rc = check_f8_size(m[0].n, m[0].k, m[0].gated != 0, who);
  if (rc) return rc;
  for (int e = 0; e < K; ++e)
    if (m[e].n != m[0].n || m[e].k != m[0].k || (m[e].gated != 0) != (m[0].gated != 0)) return set_error(MOQE_E_SHAPE, "%s: matrices of different sizes or kinds", who);
  return MOQE_OK;
}

int32_t check_f8_call(const moqe_f8_mat* experts, int32_t K, int32_t S, int32_t T, int32_t type, const char* who) {
  const int32_t rc = check_f8_experts(experts, K, who);
  if (rc) return rc;
  if (S < 0 || T < 1 || static_cast<long long>(S) * T > (1ll << 30)) return set_error(MOQE_E_SHAPE, "%s: S=%d T=%d", who, S, T);
  if (type != MOQE_TYPE_F32 && type != MOQE_TYPE_BF16 && type != MOQE_TYPE_F8) return set_error(MOQE_E_FORMAT, "%s: result of type %d", who, type);
  if (type == MOQE_TYPE_F8 && !experts[0].gated) return set_error(MOQE_E_FORMAT, "%s: only gated pairs give rows in 8 bits", who);
  if (type == MOQE_TYPE_F8 && experts[0].n > 32768) return set_error(MOQE_E_SHAPE, "%s: rows in 8 bits of %d features, at most 32768", who, experts[0].n);
  return MOQE_OK;
}

}  // namespace

int32_t check_f8_rows(const moqe_f8_rows* r, int32_t d, const char* what, const char* who) {
  if (!r) return set_error(MOQE_E_NULL, "%s: %s is NULL", who, what);
  if (!r->codes || !r->scales) return set_error(MOQE_E_NULL, "%s: codes or scales of %s are NULL", who, what);
  if (!aligned(r->codes, 16) || !aligned(r->scales, 4) || r->code_stride % 16 || r->scale_stride % 4)
    return set_error(MOQE_E_SHAPE, "%s: %s: codes must be 16-byte aligned with a stride that is a multiple of 16, scales 4-byte aligned with one of 4", who, what);
  const int blocks = f8_blocks(d);
  if (r->code_stride < static_cast<int64_t>(blocks) * F8_BLOCK || r->scale_stride < blocks || r->code_stride > (1ll << 32) || r->scale_stride > (1ll << 32))
    return set_error(MOQE_E_SHAPE, "%s: %s: strides of %lld and %lld bytes, rows of %d features have %d blocks", who, what, static_cast<long long>(r->code_stride),
                     static_cast<long long>(r->scale_stride), d, blocks);
  return MOQE_OK;
}

}  // namespace moqe

using namespace moqe;

extern "C" {

size_t moqe_f8_packed_bytes(int32_t n, int32_t k, int32_t gated) {
  return check_f8_size(n, k, gated != 0, "moqe_f8_packed_bytes") ? 0 : f8_packed(n, k, gated != 0).total;
}

int32_t moqe_f8_pack(const moqe_f8_rows* w, const moqe_f8_rows* up, int32_t n, int32_t k, void* packed, size_t bytes, void* stream) {
  const char* who = "moqe_f8_pack";
  int32_t rc = check_f8_size(n, k, up != nullptr, who);
  if (!rc) rc = check_f8_rows(w, k, "w", who);
  if (!rc && up) rc = check_f8_rows(up, k, "up", who);
  if (rc) return rc;
  if (!packed) return set_error(MOQE_E_NULL, "%s: packed is NULL", who);
  if (!aligned(packed, 256)) return set_error(MOQE_E_SHAPE, "%s: packed must be 256-byte aligned", who);
  const size_t need = f8_packed(n, k, up != nullptr).total;
  if (bytes < need) return set_error(MOQE_E_SHAPE, "%s: %zu bytes, the matrix takes %zu", who, bytes, need);
  if (dry_run()) return MOQE_OK;
  return launch_f8_pack(*w, up, n, k, static_cast<uint8_t*>(packed), static_cast<hipStream_t>(stream));
}

int32_t moqe_f8_unpack(const moqe_f8_mat* m, const moqe_f8_rows* w, const moqe_f8_rows* up, void* stream) {
  const char* who = "moqe_f8_unpack";
  int32_t rc = check_f8_experts(m, 1, who);
  if (rc) return rc;
  if (!m->packed) return set_error(MOQE_E_NULL, "%s: packed is NULL", who);
  if (!aligned(m->packed, 256)) return set_error(MOQE_E_SHAPE, "%s: packed must be 256-byte aligned", who);
  if ((m->gated != 0) != (up != nullptr)) return set_error(MOQE_E_FORMAT, "%s: up is of gated pairs, and they need it", who);
  rc = check_f8_rows(w, m->k, "w", who);
  if (!rc && up) rc = check_f8_rows(up, m->k, "up", who);
  if (rc || dry_run()) return rc;
  return launch_f8_unpack(*m, *w, up, static_cast<hipStream_t>(stream));
}

size_t moqe_f8_gemm_workspace_bytes(const moqe_f8_mat* experts, int32_t K, int32_t S, int32_t T, int32_t y_type) {
  if (check_f8_call(experts, K, S, T, y_type, "moqe_f8_gemm_workspace_bytes")) return 0;
  return f8_gemm_ws_bytes(static_cast<long long>(S) * T, experts[0].n, experts[0].k, K, experts[0].gated != 0, y_type == MOQE_TYPE_F8);
}

int32_t moqe_f8_gemm(const moqe_f8_rows* a, const int32_t* offsets, const int32_t* perm, int32_t S, int32_t T, const moqe_f8_mat* experts, int32_t K,
                     const moqe_f8_result* y, int32_t flags, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "moqe_f8_gemm";
  if (!y) return set_error(MOQE_E_NULL, "%s: y is NULL", who);
  int32_t rc = check_f8_call(experts, K, S, T, y->type, who);
  if (rc) return rc;
  if (flags & ~(MOQE_SCATTER_OUTPUT | MOQE_INPUT_IN_BUCKET_ORDER | MOQE_FAST_SUMS)) return set_error(MOQE_E_FORMAT, "%s: flags %d", who, flags);
  if (!offsets && K != 1) return set_error(MOQE_E_NULL, "%s: offsets is NULL with %d experts", who, K);
  if ((flags & MOQE_SCATTER_OUTPUT) && !perm) return set_error(MOQE_E_NULL, "%s: perm is NULL, results cannot be scattered", who);
  if (!aligned(offsets, 4) || !aligned(perm, 4)) return set_error(MOQE_E_SHAPE, "%s: misaligned offsets or perm", who);
  if (S == 0) return MOQE_OK;
  const int n = experts[0].n, k = experts[0].k;
  const long long M = static_cast<long long>(S) * T;
  rc = check_f8_rows(a, k, "a", who);
  if (rc) return rc;
  if (M * a->code_stride >= (1ll << 32) || M * a->scale_stride >= (1ll << 32)) return set_error(MOQE_E_SHAPE, "%s: %lld rows of %lld bytes exceed 4 GiB", who, M,
                                                                                                  static_cast<long long>(a->code_stride));
  for (int e = 0; e < K; ++e) {
    if (!experts[e].packed) return set_error(MOQE_E_NULL, "%s: a packed matrix is NULL", who);
    if (!aligned(experts[e].packed, 256)) return set_error(MOQE_E_SHAPE, "%s: packed matrices must be 256-byte aligned", who);
  }
  if (y->type == MOQE_TYPE_F8) {
    rc = check_f8_rows(&y->rows8, n, "rows8", who);
    if (rc) return rc;
  } else {
    const size_t size = y->type == MOQE_TYPE_F32 ? 4 : 2;
    if (!y->data) return set_error(MOQE_E_NULL, "%s: the result's data is NULL", who);
    if (!aligned(y->data, size) || y->stride < n || y->stride > (1ll << 32)) return set_error(MOQE_E_SHAPE, "%s: result rows misaligned or with stride %lld", who,
                                                                                              static_cast<long long>(y->stride));
  }
  const bool gated = experts[0].gated != 0;
  const size_t need = f8_gemm_ws_bytes(M, n, k, K, gated, y->type == MOQE_TYPE_F8);
  if (need && (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
    return set_error(MOQE_E_WORKSPACE, "%s: workspace needs %zu bytes, 256-byte aligned", who, need);
  const F8Packed p = f8_packed(n, k, gated);
  F8Args g{};
  g.a = a->codes; g.a_scales = a->scales; g.a_stride = uint32_t(a->code_stride); g.as_stride = uint32_t(a->scale_stride);
  for (int e = 0; e < K; ++e) g.w[e] = static_cast<const uint8_t*>(experts[e].packed);
  g.offsets = offsets;
  g.a_perm = (flags & MOQE_INPUT_IN_BUCKET_ORDER) ? nullptr : perm;
  g.y_perm = (flags & MOQE_SCATTER_OUTPUT) ? perm : nullptr;
  g.exact = !(flags & MOQE_FAST_SUMS);
  g.S = S; g.T = T; g.K = K; g.n = n; g.tiles = p.tiles; g.blocks = p.blocks; g.groups = p.groups; g.scale_off = uint32_t(p.scale_off);
  if (y->type == MOQE_TYPE_F8) {
    g.y8 = y->rows8.codes; g.y8_scales = y->rows8.scales; g.y8_stride = y->rows8.code_stride; g.y8_scale_stride = y->rows8.scale_stride;
  } else {
    g.y = y->data; g.y_stride = y->stride; g.y_bf16 = y->type == MOQE_TYPE_BF16;
  }
  const long long wgs = f8_work_groups(f8_shape(M, K, g.tiles, gated, g.exact), M, K, g.tiles);
  if (wgs > F8_MAX_WGS) return set_error(MOQE_E_SHAPE, "%s: %lld work-groups", who, wgs);
  if (dry_run()) return MOQE_OK;
  return launch_f8_gemm(g, gated, workspace, static_cast<hipStream_t>(stream));
}

size_t moqe_sample_workspace_bytes(int32_t S, int32_t V) {
  if (S < 1 || V < 1 || V > (1 << 20)) return 0;
  return sample_ws_bytes(S, V);
}

int32_t moqe_sample(const void* logits, int32_t type, int64_t stride, int32_t S, int32_t V, const moqe_sampling* how, const float* u, int32_t* tokens, float* logprobs,
                    void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "moqe_sample";
  if (S < 0 || V < 1 || V > (1 << 20) || S > 65535) return set_error(MOQE_E_SHAPE, "%s: %d rows (at most 65535) of %d logits (at most 2^20)", who, S, V);
  if (type != MOQE_TYPE_F32 && type != MOQE_TYPE_BF16) return set_error(MOQE_E_FORMAT, "%s: logits of type %d", who, type);
  if (!how) return set_error(MOQE_E_NULL, "%s: how is NULL", who);
  if (!aligned(how->temperature, 4) || !aligned(how->top_k, 4) || !aligned(how->top_p, 4) || !aligned(how->min_p, 4))
    return set_error(MOQE_E_SHAPE, "%s: misaligned temperature, top_k, top_p or min_p", who);
  if (S == 0) return MOQE_OK;
  if (!logits || !u || !tokens) return set_error(MOQE_E_NULL, "%s: logits, u or tokens is NULL", who);
  if (!aligned(logits, type == MOQE_TYPE_F32 ? 4 : 2) || !aligned(u, 4) || !aligned(tokens, 4) || !aligned(logprobs, 4))
    return set_error(MOQE_E_SHAPE, "%s: a pointer is not aligned to its type", who);
  if (stride < V || stride > (1ll << 32)) return set_error(MOQE_E_SHAPE, "%s: stride %lld of rows of %d logits", who, static_cast<long long>(stride), V);
  const size_t need = sample_ws_bytes(S, V);
  if (need && (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
    return set_error(MOQE_E_WORKSPACE, "%s: workspace needs %zu bytes, 256-byte aligned", who, need);
  if (dry_run()) return MOQE_OK;
  return launch_sample(logits, type == MOQE_TYPE_BF16, stride, S, V, *how, u, tokens, logprobs, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
