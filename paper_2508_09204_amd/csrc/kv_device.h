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
  const int len = b.kv_len[s];
  q.row0 = s * b.T;
  q.n = b.T;
  if (b.cu_rows) {
    const int c0 = b.cu_rows[s], c1 = b.cu_rows[s + 1];
    q.row0 = min(max(c0, 0), b.M);
    q.n = max(min(max(c1, 0), b.M) - q.row0, 0);
  }
  q.len = static_cast<int>(min(static_cast<long long>(max(len, 0)), static_cast<long long>(b.width) << bt_log2));
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
typedef float kv_f32x16 __attribute__((ext_vector_type(16)));

// Four and eight codes times their scale, exact in bf16: the scale is a power of two and the conversion takes it along.
__device__ __forceinline__ uint2 kv_four(uint32_t w, float scale) {
  return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true)));
}
__device__ __forceinline__ kv_bf16x8 kv_operand(uint32_t lo, uint32_t hi, float scale) {
  union { kv_bf16x2 p[4]; kv_bf16x8 v; } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return u.v;
}

__device__ __forceinline__ uint32_t kv_pair(float lo, float hi) {          // two bf16, to nearest even
  const __bf16 l = static_cast<__bf16>(lo), h = static_cast<__bf16>(hi);
  return uint32_t(__builtin_bit_cast(uint16_t, l)) | uint32_t(__builtin_bit_cast(uint16_t, h)) << 16;
}

// Adds eight bf16 weights to a sum in fp32, two an instruction.  The sum is of the weights as they multiply the values, so that their rounding partly cancels.
__device__ __forceinline__ float kv_add8(kv_bf16x8 w, float sum) {
  union { kv_bf16x8 v; kv_bf16x2 p[4]; } u;
  u.v = w;
  const kv_bf16x2 ones = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
#pragma unroll
  for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_fdot2_f32_bf16(u.p[i], ones, sum, false);
  return sum;
}

// Waits until no more than the N youngest loads are under way.
template <int N>
__device__ __forceinline__ void kv_wait_loads() { __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70); }

// What turns q . k into the score's base-2 exponent, and who sees what.
struct KvScore {
  const float* slopes; const int32_t* prefix;
  float scale2;                              // scale * log2 e
  float cap2, turn, of_cap;                  // cap * log2 e (0: none), 2 log2 e * scale / cap, scale / cap
  int window;
};
constexpr float KV_LOG2E = 1.4426950408889634f;
inline bool kv_capped(const moqe_attention& a) { return a.cap > 0.f && a.cap < INFINITY; }      // an infinite cap is none
inline KvScore kv_score(const moqe_attention& a, const moqe_kv_batch& b, const moqe_kv_cache& c) {
  const bool capped = kv_capped(a);
  return KvScore{a.slopes, a.prefix, a.scale * KV_LOG2E, capped ? a.cap * KV_LOG2E : 0.f, capped ? 2.f * KV_LOG2E * a.scale / a.cap : 0.f,
                 capped ? a.scale / a.cap : 0.f,
                 kv_window(a.window, static_cast<long long>(b.table_width) * c.block_tokens)};
}
// What a score needs beyond its scale: KV_CAP, KV_BIAS (by distance; also where the scale is not positive, since the kernels take the largest product for the largest score).
// KV_FAR_CAP: both, for caps past KV_NEAR_CAP.
enum : int { KV_PLAIN = 0, KV_CAP = 1, KV_BIAS = 2, KV_FAR_CAP = 7 };
// cap * tanh(x / cap) is cap * (1 - 2 / (1 + e^(2 x / cap))), whose error is some 2^-22 of cap, wherever x lies: up to a cap of 2^10 that moves a weight by no more than 2^-12 of it, a
// sixteenth of what its rounding to bf16 does.  For larger caps the power series takes over where x lies below an eighth of the cap, x (1 - z^2 / 3 + 2 z^4 / 15) for z = x / cap,
// which leaves 2^-22 of x.  Those are kernels of their own: with the series in all, prompts of capped scores take 1.1 to 1.3 times as long (24 x up to 700 rows, heads of 64, 102 -> 135 us).
constexpr float KV_NEAR_CAP = 1024.f;
inline int kv_extra(const moqe_attention& a) {
  const bool capped = kv_capped(a);
  if (capped && a.cap > KV_NEAR_CAP) return KV_FAR_CAP;
  return (capped ? KV_CAP : 0) | (a.slopes || (!capped && !(a.scale > 0.f)) ? KV_BIAS : 0);
}
// From the product d = q . k.
template <int EXTRA>
__device__ __forceinline__ float kv_extra_score(const KvScore& sc, float d, float slope, float distance) {
  float v = d * sc.scale2;
  if constexpr ((EXTRA & KV_CAP) != 0) {
    const float z = d * sc.of_cap, zz = z * z, series = v * fmaf(zz, fmaf(zz, 2.f / 15, -1.f / 3), 1.f);
    v = fmaf(-2.f * sc.cap2, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(d * sc.turn)), sc.cap2);
    if (EXTRA == KV_FAR_CAP && zz < 1.f / 64) v = series;
  }
  if constexpr ((EXTRA & KV_BIAS) != 0) v = fmaf(-slope, fabsf(distance), v);
  return v;
}

// Bytes of NaN among four codes, as 1 in their lowest bits.
__device__ __forceinline__ uint32_t kv_nan_bytes(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7; }
__device__ __forceinline__ uint32_t kv_nan_bytes(uint4 w) { return kv_nan_bytes(w.x) | kv_nan_bytes(w.y) | kv_nan_bytes(w.z) | kv_nan_bytes(w.w); }
__device__ __forceinline__ uint4 kv_without_nan(uint4 w) {
  return make_uint4(w.x & ~(kv_nan_bytes(w.x) * 0xffu), w.y & ~(kv_nan_bytes(w.y) * 0xffu), w.z & ~(kv_nan_bytes(w.z) * 0xffu),
                    w.w & ~(kv_nan_bytes(w.w) * 0xffu));
}

// A lane's 16 bytes of values (tokens t .. t + 3 and t + 16 .. t + 19 of two dims) with those from token `end` on, which nobody sees, as zeros.
__device__ __forceinline__ uint4 kv_before(uint4 w, int t, int end) {
  auto mask = [](int n) { return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1u; };
  const uint32_t a = mask(end - t), b = mask(end - t - 16);
  return make_uint4(w.x & a, w.y & b, w.z & a, w.w & b);
}

// Parts of rows, to be joined.
struct KvParts {
  float2* ml; float* o;         // [part][..] maximum and sum, [..][head_dim] rows that are not divided by the sum; NULL: there is one part
};
inline KvParts kv_parts(void* ws, size_t rows) {
  return KvParts{static_cast<float2*>(ws), reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + align256(rows * 8))};
}

}  // namespace moqe
