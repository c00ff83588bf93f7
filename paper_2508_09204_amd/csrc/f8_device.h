// Device helpers of the 8-bit floating-point rows.
#pragma once

#include "f8_rows.h"
#include "moqe_internal.h"

#include <type_traits>

namespace moqe {

typedef int f8_i32x8 __attribute__((ext_vector_type(8)));
typedef float f8_f32x4 __attribute__((ext_vector_type(4)));

// Scale exponent for values whose largest finite size is `top`.
__device__ __forceinline__ int f8_exponent(float top) { return kv_scale_exponent(__float_as_uint(top)); }

// Eight codes of x * 2^-e, to nearest even.  |x| <= 448 * 2^e but for infinities, which the conversion would make NaN of: they become the largest code.  448 * 2^120 is an infinity itself: values
// of that scale are halved first, by which only those that are zeros in it lose digits.
__device__ __forceinline__ uint2 f8_codes(const float* x, int e) {
  const bool far = e > 119;
  const float scale = __uint_as_float(uint32_t(e - far + 127) << 23), most = 448.f * scale;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fabsf(x[i]) == INFINITY ? copysignf(most, x[i]) : x[i] * (far ? 0.5f : 1.f);
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  s16x2 lo = {0, 0}, hi = {0, 0};
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, v[0], v[1], scale, false);
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, v[2], v[3], scale, true);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, v[4], v[5], scale, false);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, v[6], v[7], scale, true);
  return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}

// Largest finite size of eight values; NaN is passed over.
__device__ __forceinline__ float f8_top(const float* x, float top = 0.f) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(x[i]);
    top = a < INFINITY ? fmaxf(top, a) : top;
  }
  return top;
}

// The largest of 16 neighbouring lanes (not negative), in all of them.
__device__ __forceinline__ float f8_row_top(float x) {
  auto turned = [](float v, auto ctrl) { return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, false)); };
  x = fmaxf(x, turned(x, std::integral_constant<int, 0x121>()));      // row_ror:1, 2, 4, 8
  x = fmaxf(x, turned(x, std::integral_constant<int, 0x122>()));
  x = fmaxf(x, turned(x, std::integral_constant<int, 0x124>()));
  return fmaxf(x, turned(x, std::integral_constant<int, 0x128>()));
}

// What the launch of a grouped product knows.
struct F8Args {
  const uint8_t *a, *a_scales;
  const uint8_t* w[MOQE_MAX_EXPERTS];
  const int32_t *offsets, *a_perm, *y_perm;      // offsets NULL: one expert, all rows
  void* y; uint8_t *y8, *y8_scales;              // y, or rows in 8 bits
  long long y_stride, y8_stride, y8_scale_stride;
  uint32_t a_stride, as_stride;                  // bytes
  int32_t S, T, K, n, tiles, blocks, groups;
  uint32_t scale_off;
  int32_t y_bf16, exact;                         // exact: fp32 sums of exact products
};
// Bucket of an expert in rows: first row and number.  Device values are taken into their ranges.
__device__ __forceinline__ int2 f8_bucket(const F8Args& a, int e) {
  if (!a.offsets) return make_int2(0, a.S * a.T);
  const int c0 = min(max(a.offsets[e], 0), a.S), c1 = min(max(a.offsets[e + 1], c0), a.S);
  return make_int2(c0 * a.T, (c1 - c0) * a.T);
}
// Row of bucket row m in the caller's order, -1 where perm names no sample.
__device__ __forceinline__ int f8_row(const F8Args& a, const int32_t* perm, int m) {
  if (!perm) return m;
  const int slot = m / a.T, s = perm[slot];
  return s < 0 || s >= a.S ? -1 : s * a.T + (m - slot * a.T);
}

__device__ __forceinline__ uint32_t f8_bf16_pair(float lo, float hi) {
  const __bf16 l = static_cast<__bf16>(lo), h = static_cast<__bf16>(hi);
  return uint32_t(__builtin_bit_cast(uint16_t, l)) | uint32_t(__builtin_bit_cast(uint16_t, h)) << 16;
}
// Four values of a row from column n0 on.  Wide stores need no alignment beyond an element's.
__device__ __forceinline__ void f8_store(const F8Args& a, int row, int n0, f8_f32x4 v) {
  const long long at = row * a.y_stride + n0;
  if (n0 + 4 <= a.n) {
    const uint2 h = make_uint2(f8_bf16_pair(v[0], v[1]), f8_bf16_pair(v[2], v[3]));
    if (a.y_bf16) __builtin_memcpy(static_cast<uint16_t*>(a.y) + at, &h, 8);
    else __builtin_memcpy(static_cast<float*>(a.y) + at, &v, 16);
    return;
  }
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (n0 + i < a.n) {
      if (a.y_bf16) static_cast<uint16_t*>(a.y)[at + i] = uint16_t(f8_bf16_pair(v[i], 0.f));
      else static_cast<float*>(a.y)[at + i] = v[i];
    }
}
// silu(g) * u in fp32: g / (1 + 2^y) * u, y = -log2(e) g, with the hardware's exponential and reciprocal, nine half steps or 2^-20.8 of the result (2^-22.2 measured) for g > -87, from where on it is within 2^-119 of u.  What the rounded y lacks grows with
// |g| and is made up for behind the exponential (it would be 2^-18 of the result at g = -60).
__device__ __forceinline__ float f8_gated(float g, float u) {
  const float y = -1.44269502f * g, lost = fabsf(g) < 128.f ? fmaf(-1.44269502f, g, -y) - 1.92596303e-8f * g : 0.f;
  return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(y) * fmaf(lost, 0.69314718f, 1.f)) * u;
}

typedef int f8_i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 f8_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 f8_bf16x8 __attribute__((ext_vector_type(8)));
union F8Frag { f8_i32x4 u[2]; f8_i32x8 v; };         // a lane's 32 codes of an operand's block of 128

// acc += a block of 128: weights (16 features) times activations (16 rows), scales in byte J of each lane's dword; lane 16 q + r gets features 4 q .. 4 q + 3 of row r.
template <int J>
__device__ __forceinline__ f8_f32x4 f8_mfma(const F8Frag& w, const F8Frag& x, const f8_f32x4& c, uint32_t ws, uint32_t xs) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.v, x.v, c, 0, 0, J, int(ws), J, int(xs));
}

// That instruction adds 8 neighbouring columns at a time, each product cut to 2^-13 of the largest one's power of two: 1.8e-5 of the result in the mean square for normal operands, which is
// 200 times what fp32 sums do, and more than a rounding to bf16 for results far below the others.  So products of bf16, at half the rate, unless the caller asks for the fast ones: codes times
// their scale are exact there.
__device__ __forceinline__ float f8_scale(uint32_t byte) { return __uint_as_float((byte & 255) << 23); }
__device__ __forceinline__ f8_bf16x8 f8_exact(uint32_t lo, uint32_t hi, float scale) {
  union { f8_bf16x2 p[4]; f8_bf16x8 v; } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return u.v;
}
// Quarter j of an operand: eight codes of each lane, an operand of a 16x16x32 product.
__device__ __forceinline__ f8_bf16x8 f8_quarter(const F8Frag& f, int j, float scale) { return f8_exact(uint32_t(f.v[2 * j]), uint32_t(f.v[2 * j + 1]), scale); }

__device__ __forceinline__ __amdgpu_buffer_rsrc_t f8_rsrc(const uint8_t* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, int(bytes), 0x00020000);   // raw buffer, 32-bit data format
}
enum F8Out : int { F8_PLAIN = 0, F8_GATED = 1, F8_GATED8 = 2 };

}  // namespace moqe
