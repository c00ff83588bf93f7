// Where things lie in the 8-bit key/value cache and how its attention is divided, in plain C++ (a host compiler can check it).
#pragma once

#include <stddef.h>
#include <stdint.h>

#ifdef __HIPCC__
#include <hip/hip_runtime.h>
#define MOQE_HD __host__ __device__ __forceinline__
#else
#define MOQE_HD inline
#endif

namespace moqe {

// Byte of (token, dim) among the codes of one block and head.  The orders are those of 16x16x32 matrix-core operands: a lane's 8 bytes of a step are
// its operand, 16 bytes cover two steps.  Keys are the rows of the first product, S^T = K Q^T, whose result leaves lane 16 kq + r
// with tokens 4 kq .. 4 kq + 3 of 16 for query r; two such results are the operand of the second, O^T = V^T P^T, without any
// exchange between lanes, if the values' operand takes its 8 tokens of 32 in the same order: 4 kq + i, then 16 + 4 kq + i.
MOQE_HD uint32_t kv_key_at(uint32_t token, uint32_t dim, uint32_t dh) {
  const uint32_t lane = (dim % 32) / 8 * 16 + token % 16;
  return token / 16 * (16 * dh) + dim / 64 * 1024 + lane * 16 + dim % 64 / 32 * 8 + dim % 8;
}
MOQE_HD uint32_t kv_value_at(uint32_t token, uint32_t dim, uint32_t dh) {
  const uint32_t u = token % 32, lane = u % 16 / 4 * 16 + dim % 16;
  return token / 32 * (32 * dh) + dim / 32 * 1024 + lane * 16 + dim % 32 / 16 * 8 + u / 16 * 4 + u % 4;
}

// Exponent of the smallest power of two s with amax <= 448 s, in [-120, 120]: 448 = 1.75 * 2^8.  bits: those of amax (finite, not negative).
MOQE_HD int kv_scale_exponent(uint32_t bits) {
  const int e = int(bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
  return e < -120 ? -120 : e > 120 ? 120 : e;
}

// The window that kernels work with.  One as long as a sequence can be (`tokens`, 2^30 at most) hides nothing: none then.  So the first position of a call's rows (-2^24 at least)
// less a window stays in 32 bits, here and below.
inline int kv_window(int window, long long tokens) { return window > 0 && window < tokens ? window : 0; }

// Tokens that every row sees: a device value, taken into its range.
MOQE_HD int kv_prefix(int prefix, int len) { return prefix < 0 ? 0 : prefix < len ? prefix : len; }

// Steps of 32 tokens that the rows at positions first_pos .. of a sequence with len tokens go through: steps of the prefix, then steps from the window's
// first token on.  Step number j of `count` is tokens 32 * step(j) ...
struct KvSteps {
  int pre, skip, count;        // steps before the gap, steps of the gap, steps in all
  MOQE_HD int step(int j) const { return j < pre ? j : j + skip; }
};
MOQE_HD KvSteps kv_steps(int len, int seen, int first_pos, int window, int prefix) {   // seen: tokens below which anything is seen, <= len
  KvSteps k;
  const int all = (seen + 31) / 32;
  int lo = window > 0 ? first_pos + 1 - window : 0;
  lo = lo < 0 ? 0 : lo;
  const int from = lo / 32 < all ? lo / 32 : all;
  int pre = (kv_prefix(prefix, len) + 31) / 32;
  pre = pre < all ? pre : all;
  k.pre = pre < from ? pre : from;
  k.skip = from - k.pre;
  k.count = all - k.skip;
  return k;
}

// What a row at position p sees: tokens below `pre` and `span` tokens from `lo` on.
struct KvSight {
  int lo;
  uint32_t span;
  MOQE_HD bool sees(int t, int pre) const { return uint32_t(t - lo) < span || t < pre; }
};
MOQE_HD KvSight kv_sight(int p, int len, int window) {
  const int hi = len < p + 1 ? len : p + 1, from = window > 0 ? p - window + 1 : 0, lo = from > 0 ? from : 0;
  return KvSight{lo, uint32_t(hi > lo ? hi - lo : 0)};
}
// First tokens t0 of 32-token steps that rows at positions p0 .. p1 see all of, or may see any of.
struct KvRange {
  int lo, hi, pre;
  MOQE_HD bool has(int t0) const { return (t0 >= lo && t0 < hi) || t0 < pre; }
};
MOQE_HD KvRange kv_all_see(int p0, int p1, int pre, int window) { return KvRange{window > 0 ? p1 - window + 1 : 0, p0 - 30, pre - 31}; }
MOQE_HD KvRange kv_some_see(int p0, int p1, int pre, int window) { return KvRange{window > 0 ? p0 - window - 30 : 0, p1 + 1, pre}; }

}  // namespace moqe
