// Tokens from logits by temperature, top-k, top-p and min-p.
#include "moqe_internal.h"

namespace moqe {

struct SampleArgs {
  const void* logits; long long stride;
  const float* temperature; const int32_t* top_k; const float *top_p, *min_p; const float* u;
  int32_t* tokens; float* logprobs;
  int S, V;
};

// A finite or plus infinite value as an integer of the same order, not 0; 0 for minus infinity and NaN.
__device__ __forceinline__ uint32_t sample_key(float x) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(x + 0.f);                // -0 as +0
  return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float sample_value(uint32_t key) { return __uint_as_float((key >> 31) ? key & 0x7fffffffu : ~key); }

constexpr double SAMPLE_ONE = double(1ull << 42);             // a weight of 1

// One work-group a row; the cut between kept and dropped is found by bisection over keys, each step a pass over the row.
template <bool BF16>
__global__ __launch_bounds__(1024) void k_sample_simple(SampleArgs a) {
  __shared__ unsigned long long part[16];
  __shared__ uint32_t tops[16];
  const int s = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, V = a.V;
  const char* base = static_cast<const char*>(a.logits) + s * a.stride * (BF16 ? 2 : 4);
  auto key = [&](int i) {
    if constexpr (BF16) return sample_key(__uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(base)[i]) << 16));
    else return sample_key(reinterpret_cast<const float*>(base)[i]);
  };
  auto total = [&](auto&& of) {                               // sum of of(i) over the row, in all threads
    unsigned long long v = 0;
    for (int i = tid; i < V; i += 1024) v += of(i);
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if (lane == 0) part[wave] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < 16; ++w) v += part[w];
    return v;
  };
  uint32_t top = 0;
  for (int i = tid; i < V; i += 1024) top = max(top, key(i));
  for (int d = 32; d >= 1; d >>= 1) top = max(top, uint32_t(__shfl_xor(int(top), d)));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  for (int w = 0; w < 16; ++w) top = max(top, tops[w]);
  if (top == 0) {
    if (tid == 0) { a.tokens[s] = -1; if (a.logprobs) a.logprobs[s] = -INFINITY; }
    return;
  }
  const float largest = sample_value(top);
  const float T = a.temperature ? a.temperature[s] : 1.f;
  const bool greedy = !(T > 0.f);
  auto weight = [&](uint32_t k) {
    if (k == top) return 1.0;
    if (k == 0 || largest == INFINITY) return 0.0;
    return exp((double(sample_value(k)) - double(largest)) / (greedy ? 1.0 : double(T)));
  };
  auto mass = [&](uint32_t k) { return static_cast<unsigned long long>(rint(weight(k) * SAMPLE_ONE)); };
  // kept: keys above `cut`, and the first `ties` of those equal to it
  uint32_t cut = 1;
  unsigned long long ties = ~0ull;
  long long k = a.top_k ? a.top_k[s] : 0;
  if (greedy) k = 1;
  auto bisect = [&](auto&& reached) {                          // largest key with reached(key), which holds for 1
    uint32_t lo = 1, hi = top;
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo + 1) / 2;
      if (reached(mid)) lo = mid; else hi = mid - 1;
    }
    return lo;
  };
  if (k > 0) {
    const unsigned long long all = total([&](int i) { return key(i) != 0 ? 1ull : 0ull; });
    if (static_cast<unsigned long long>(k) < all) {
      cut = bisect([&](uint32_t c) { return total([&](int i) { return key(i) >= c ? 1ull : 0ull; }) >= static_cast<unsigned long long>(k); });
      ties = k - total([&](int i) { return key(i) > cut ? 1ull : 0ull; });
    }
  }
  const unsigned long long equal = total([&](int i) { return key(i) == cut ? 1ull : 0ull; });
  if (ties > equal) ties = equal;
  const float p = a.top_p ? a.top_p[s] : 1.f;
  auto above = [&](uint32_t c) { return total([&](int i) { const uint32_t x = key(i); return x > c ? mass(x) : 0ull; }); };
  if (p < 1.f) {
    const double want = double(p > 0.f ? p : 0.f) * double(above(cut) + ties * mass(cut));
    // a token is kept while the weight ahead of it is less than `want` (and the first one always)
    const uint32_t c = bisect([&](uint32_t x) { return x <= cut || double(above(x - 1 < cut ? cut : x - 1)) >= want; });
    if (c > cut) {
      cut = c;
      ties = total([&](int i) { return key(i) == cut ? 1ull : 0ull; });
    }
    const double left = want - double(above(cut)), each = double(mass(cut));
    unsigned long long need = left > 0. && each > 0. ? static_cast<unsigned long long>(ceil(left / each)) : cut == top ? 1 : 0;
    if (cut == top && need < 1) need = 1;
    if (left > 0. && need < ties) ties = need;
    else if (!(left > 0.)) ties = need;
  }
  float least = a.min_p ? a.min_p[s] : 0.f;
  least = least > 1.f ? 1.f : least;
  // the ties are the first ones by index: a bound on the index, by bisection
  int bound = V;
  if (ties < total([&](int i) { return key(i) == cut ? 1ull : 0ull; })) {
    int lo = 0, hi = V;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (total([&](int i) { return key(i) == cut && i < mid ? 1ull : 0ull; }) >= ties) hi = mid; else lo = mid + 1;
    }
    bound = lo;
  }
  auto kept = [&](int i) {
    const uint32_t x = key(i);
    if (x < cut || (x == cut && i >= bound)) return 0ull;
    return least > 0.f && !(weight(x) >= double(least)) ? 0ull : mass(x);
  };
  const unsigned long long W = total(kept);
  float u = a.u[s];
  u = u > 0.f ? fminf(u, 1.f) : 0.f;
  const double goal = double(u) * double(W);
  // first index whose running weight exceeds the goal; the last one with weight if none does
  int lo = 0, hi = V - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (double(total([&](int i) { return i <= mid ? kept(i) : 0ull; })) > goal) hi = mid; else lo = mid + 1;
  }
  int token = lo;
  if (!(double(W) > goal)) {
    unsigned long long last = 0;
    for (int i = tid; i < V; i += 1024)
      if (kept(i)) last = i;
    uint32_t t = uint32_t(last);
    for (int d = 32; d >= 1; d >>= 1) t = max(t, uint32_t(__shfl_xor(int(t), d)));
    __syncthreads();
    if (lane == 0) tops[wave] = t;
    __syncthreads();
    for (int w = 0; w < 16; ++w) t = max(t, tops[w]);
    token = int(t);
  }
  if (tid == 0) {
    a.tokens[s] = token;
    if (a.logprobs) a.logprobs[s] = float(log(weight(key(token)) * SAMPLE_ONE / double(W)));
  }
}

size_t sample_ws_bytes(int, int) { return 0; }

int32_t launch_sample(const void* logits, bool bf16, long long stride, int S, int V, const moqe_sampling& how, const float* u, int32_t* tokens, float* logprobs,
                      void*, hipStream_t st) {
  const SampleArgs a{logits, stride, how.temperature, how.top_k, how.top_p, how.min_p, u, tokens, logprobs, S, V};
  ProfileScope ps(MOQE_PK_OTHER, st);
  if (bf16) hipLaunchKernelGGL(k_sample_simple<true>, dim3(S), dim3(1024), 0, st, a);
  else hipLaunchKernelGGL(k_sample_simple<false>, dim3(S), dim3(1024), 0, st, a);
  return check_launch("sample");
}

}  // namespace moqe
