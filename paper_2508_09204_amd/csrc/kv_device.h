// Device helpers shared by the kernels that write and read the 8-bit key/value cache.
#pragma once

#include "kv_cache.h"
#include "moqe_internal.h"

namespace moqe {

struct KvBatch {
  const int32_t *table, *kv_len, *cu_rows;
  int32_t S, T, M, width;
};
struct KvCache {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  int32_t n_blocks, bt_log2, heads;
};

// Where a sequence's rows lie and which positions they have.  Device values are taken into their ranges, so that bad ones read nothing outside.
struct KvSeq {
  int row0, n;                  // first row, rows (those past the first T are not computed)
  int len;                      // tokens with the new ones
  __device__ __forceinline__ int first() const { return len - n; }      // position of row 0, may be negative
};
__device__ __forceinline__ KvSeq kv_seq(const KvBatch& b, int s, int bt_log2) {
  KvSeq q;
  q.row0 = s * b.T;
  q.n = b.T;
  if (b.cu_rows) {
    const int c0 = b.cu_rows[s], c1 = b.cu_rows[s + 1];
    q.row0 = min(max(c0, 0), b.M);
    q.n = max(min(max(c1, 0), b.M) - q.row0, 0);
  }
  q.len = static_cast<int>(min(static_cast<long long>(max(b.kv_len[s], 0)), static_cast<long long>(b.width) << bt_log2));
  return q;
}

inline KvBatch kv_batch_args(const moqe_kv_batch& b) {
  return KvBatch{b.block_table, b.kv_len, b.cu_rows, b.S, b.T, b.M, b.table_width};
}
inline KvCache kv_cache_args(const moqe_kv_cache& c) {
  return KvCache{c.k, c.v, c.k_scale, c.v_scale, c.n_blocks, c.block_tokens == 32 ? 5 : c.block_tokens == 64 ? 6 : 7, c.n_heads};
}

typedef __bf16 kv_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 kv_bf16x8 __attribute__((ext_vector_type(8)));
typedef float kv_f32x4 __attribute__((ext_vector_type(4)));

// Eight codes times their scale, exact in bf16: the scale is a power of two and the conversion takes it along.
__device__ __forceinline__ kv_bf16x8 kv_operand(uint32_t lo, uint32_t hi, float scale) {
  union { kv_bf16x2 p[4]; kv_bf16x8 v; } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return u.v;
}

// What turns q . k into the score's base-2 exponent, and who sees what.
struct KvScore {
  const float* slopes; const int32_t* prefix;
  float scale, cap;                          // as the caller gave them; cap <= 0: none
  int window;
};
constexpr float KV_LOG2E = 1.4426950408889634f;

// cap * tanh(a / cap) as cap * (1 - 2 / (1 + e^(2 a / cap))): its error is some 2^-23 of cap, wherever a lies.
__device__ __forceinline__ float kv_capped(float a, float cap) {
  return cap - 2.f * cap / (1.f + exp2f(a * (2.f * KV_LOG2E) / cap));
}

__device__ __forceinline__ bool kv_sees(int t, int p, int len, int prefix, int window) {
  return t < len && (t < prefix || (t <= p && (window <= 0 || p - t < window)));
}

}  // namespace moqe
