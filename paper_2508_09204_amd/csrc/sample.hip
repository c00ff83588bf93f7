// Tokens from logits by temperature, top-k, top-p and min-p.
//
// Weights are 2^t for t = l log2(e) / T.  Everything that decides is an integer sum, so that neither the division of a row over work-groups nor the order of atomics can change a result:
// weights are counted in units of 2^(a - 43), a the first integer above the largest t, from a table of 2^(j / 256) and a cubic (2^-42 of a weight).  A chunk of a row does not know the row's
// largest logit; but it can take an integer `a` of its own, and sums of different chunks differ by a shift.
//
//   k_sample_chunks  8192 logits a work-group: their largest, sums of 256 neighbours, and (filtered rows) counts and weights of bins a quarter of an octave wide, counted down from the largest
//   k_sample_cut     filtered rows, again by chunks: the bins of the whole row give those that the cuts of top-k and top-p fall into; sums of 256 neighbours that are kept for sure, and a list
//                    of what lies in the cuts' bins
//   k_sample_draw    a work-group a row: the cuts inside their bins, by counting keys in 1024 bins, then in 1024 of the one they fall into, until a bin is one key; the neighbourhood that the
//                    running weight passes u W in; the token in it
// The logits are read once from memory, and a second time, from the caches, where there are filters.
#include "moqe_internal.h"

#include <type_traits>

namespace moqe {

constexpr int SMP_CHUNK = 8192, SMP_NEIGHBOURS = 256, SMP_BLOCKS = SMP_CHUNK / SMP_NEIGHBOURS;
constexpr int SMP_BINS = 192;                  // quarters of an octave below the largest; the last one: everything that weighs nothing (2^-47 and less)
constexpr int SMP_LIST = 8192;                 // of a row: longer lists are read from the logits instead
constexpr int SMP_ONE = 43;

typedef unsigned long long smp_u64;

struct SampleArgs {
  const void* logits; long long stride;
  const float* temperature; const int32_t* top_k; const float *top_p, *min_p; const float* u;
  int32_t* tokens; float* logprobs;
  int32_t S, V, chunks;
  struct SampleChunk* chunk; struct SampleRow* row; smp_u64* kept; uint32_t* list;       // [S][chunks], [S], [S][chunks * SMP_BLOCKS], [S][SMP_LIST]
};
struct SampleChunk {
  uint32_t top, top_at;                        // largest key and its first index; 0: nothing but minus infinity and NaN
  smp_u64 block[SMP_BLOCKS];
  smp_u64 mass[SMP_BINS];
  uint32_t count[SMP_BINS];
};
struct SampleRow {                             // where the cuts lie
  int32_t k_bin, p_lo, p_hi, listed;           // bin of the cut of top-k (SMP_BINS: none), first and last bin that the cut of top-p may lie in (none: SMP_BINS, -1), elements of those bins
  smp_u64 k_above, k_mass, p_mass;             // elements above k_bin, weight above it, weight above p_lo
};

// A value above minus infinity as an integer of the same order, not 0; 0 for minus infinity and NaN.
__device__ __forceinline__ uint32_t smp_key(float x) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(x + 0.f);                // -0 as +0
  return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float smp_value(uint32_t key) { return __uint_as_float((key >> 31) ? key & 0x7fffffffu : ~key); }
constexpr uint32_t SMP_INFINITE = 0xff800000u;                // key of plus infinity

// 2^(j / 256)
struct SmpTable { double v[256]; };
constexpr SmpTable smp_table() {
  SmpTable t{};
  for (int j = 0; j < 256; ++j) {
    const double x = j * (0.69314718055994530942 / 256);
    double term = 1, sum = 1;
    for (int i = 1; i < 22; ++i) { term = term * x / i; sum += term; }
    t.v[j] = sum;
  }
  return t;
}
__device__ constexpr SmpTable SMP_POWERS = smp_table();

// How a row's logits weigh, given the largest (of a chunk or of the row).  Differences of logits come first: they are exact or nearly so, also where t itself is far from 0.
struct SmpScale {
  double c, top_v, top_t, shift, floor4;
  bool infinite;
  uint32_t top;
  static __device__ double per_logit(float T) { return T > 0.f ? 1.4426950408889634074 / double(T) : 0.0; }
  __device__ SmpScale(double c_, uint32_t top_key) : c(c_), top(top_key) {
    infinite = top_key == SMP_INFINITE;
    top_v = infinite ? 0.0 : double(smp_value(top_key));
    top_t = top_v * c;
    shift = (top_t - anchor() + SMP_ONE) * 256;
    floor4 = floor(top_t * 4);
  }
  __device__ double anchor() const { return floor(top_t) + 1; }
  // how many units of the other (a chunk's) are one of this (the row's), as a shift; bins between their largest
  __device__ int unit_shift(const SmpScale& chunk) const {
    if (infinite || chunk.infinite) return infinite == chunk.infinite ? 0 : 64;
    const double d = anchor() - chunk.anchor();
    return d < 64 ? int(d) : 64;
  }
  __device__ int bin_shift(const SmpScale& chunk) const {
    if (infinite || chunk.infinite) return infinite == chunk.infinite ? 0 : SMP_BINS;
    const double d = floor4 - chunk.floor4;
    return d < SMP_BINS ? int(d) : SMP_BINS;
  }
  __device__ int bin(uint32_t key) const {
    if (infinite) return key == top ? 0 : SMP_BINS - 1;
    const double d = floor4 - floor(double(smp_value(key)) * c * 4);
    return d < SMP_BINS - 1 ? int(d) : SMP_BINS - 1;
  }
  __device__ double below(uint32_t key) const { return infinite ? (key == top ? 0.0 : -INFINITY) : (double(smp_value(key)) - top_v) * c; }       // log2 of its weight over the largest
  __device__ smp_u64 mass(uint32_t key, const double* powers) const {
    double u = fma(double(smp_value(key)) - top_v, c * 256, shift);       // 256 log2 of the units
    if (infinite) u = key == top ? shift : -1e6;
    if (key == 0 || !(u > -512.0)) return 0;
    const double n = rint(u), r = (u - n) * (0.69314718055994530942 / 256);
    const int i = int(n);
    const double p = fma(r, fma(r, fma(r, 1.0 / 6, 0.5), 1.0), 1.0);
    const double x = __builtin_amdgcn_ldexp(powers[i & 255] * p, i >> 8) + 4503599627370496.0;       // 2^52: the integer stands in the mantissa's last bits
    return __builtin_bit_cast(smp_u64, x) & 0xfffffffffffffull;
  }
  __device__ double units(uint32_t key) const { return below(key) + shift * (1.0 / 256); }              // log2 of its mass
};

// Sixteen logits of a thread as keys: four at each of four places, SMP_NEIGHBOURS to a wave and place.  Past the row's end: 0.
template <bool BF16>
__device__ __forceinline__ void smp_load(const SampleArgs& a, int s, int chunk, uint32_t (&key)[4][4]) {
  const char* row = static_cast<const char*>(a.logits) + s * a.stride * (BF16 ? 2 : 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = chunk * SMP_CHUNK + j * 2048 + int(threadIdx.x) * 4;
    float v[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (i + 4 <= a.V) {                                         // wide loads need no alignment beyond an element's
      if constexpr (BF16) {
        uint2 w;
        __builtin_memcpy(&w, row + i * 2ll, 8);
        v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u); v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
      } else {
        uint4 w;
        __builtin_memcpy(&w, row + i * 4ll, 16);
        v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (i + e < a.V) v[e] = BF16 ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(row)[i + e]) << 16) : reinterpret_cast<const float*>(row)[i + e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) key[j][e] = smp_key(v[e]);
  }
}
template <bool BF16>
__device__ __forceinline__ uint32_t smp_one(const SampleArgs& a, int s, int i) {
  if constexpr (BF16) return smp_key(__uint_as_float(uint32_t(static_cast<const uint16_t*>(a.logits)[s * a.stride + i]) << 16));
  else return smp_key(static_cast<const float*>(a.logits)[s * a.stride + i]);
}

__device__ __forceinline__ smp_u64 smp_wave_sum(smp_u64 v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ smp_u64 smp_wave_upto(smp_u64 v) {      // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const smp_u64 o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// What is asked of a row.
struct SmpAsk {
  float T, p, least;
  int k;                             // 0: all
  bool greedy, filtered;
  __device__ SmpAsk(const SampleArgs& a, int s) {
    T = a.temperature ? a.temperature[s] : 1.f;
    greedy = !(T > 0.f);
    k = a.top_k ? a.top_k[s] : 0;
    if (k < 1 || k >= a.V) k = 0;
    p = a.top_p ? a.top_p[s] : 1.f;
    if (!(p < 1.f)) p = 1.f;
    if (!(p > 0.f)) p = 0.f;
    least = a.min_p ? a.min_p[s] : 0.f;
    least = least > 0.f ? fminf(least, 1.f) : 0.f;
    filtered = !greedy && (k > 0 || p < 1.f || least > 0.f);
  }
};

// Largest key of the row, by all lanes of a wave.
__device__ __forceinline__ uint32_t smp_row_top(const SampleArgs& a, int s) {
  uint32_t top = 0;
  for (int c = threadIdx.x & 63; c < a.chunks; c += 64) top = max(top, a.chunk[static_cast<size_t>(s) * a.chunks + c].top);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) top = max(top, uint32_t(__shfl_xor(int(top), d)));
  return top;
}

template <bool BF16>
__global__ __launch_bounds__(512) void k_sample_chunks(SampleArgs a) {
  __shared__ double powers[256];
  __shared__ uint32_t tops[8], count[SMP_BINS];
  __shared__ int at[8];
  __shared__ smp_u64 mass[SMP_BINS];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, s = blockIdx.y, chunk = blockIdx.x;
  SampleChunk& out = a.chunk[static_cast<size_t>(s) * a.chunks + chunk];
  uint32_t key[4][4];
  smp_load<BF16>(a, s, chunk, key);
  if (tid < 256) powers[tid] = SMP_POWERS.v[tid];
  const SmpAsk ask(a, s);
  for (int b = tid; b < SMP_BINS; b += 512) { count[b] = 0; mass[b] = 0; }
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, key[j][e]);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) top = max(top, uint32_t(__shfl_xor(int(top), d)));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) top = max(top, tops[w]);
  if (ask.greedy) {                            // the first index of the largest
    int first = 1 << 30;
#pragma unroll
    for (int j = 3; j >= 0; --j)
#pragma unroll
      for (int e = 3; e >= 0; --e)
        if (key[j][e] == top) first = chunk * SMP_CHUNK + j * 2048 + tid * 4 + e;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) first = min(first, __shfl_xor(first, d));
    if (lane == 0) at[wave] = first;
    __syncthreads();
    if (tid == 0) {
#pragma unroll
      for (int w = 0; w < 8; ++w) first = min(first, at[w]);
      out.top = top;
      out.top_at = uint32_t(first);
    }
    return;
  }
  if (tid == 0) out.top = top;
  if (top == 0) return;
  const double per = SmpScale::per_logit(ask.T);
  const SmpScale sc(per, top);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    smp_u64 sum = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const smp_u64 m = sc.mass(key[j][e], powers);
      sum += m;
      if (ask.filtered && key[j][e] != 0) {
        const int b = sc.bin(key[j][e]);
        atomicAdd(&count[b], 1u);
        if (m) atomicAdd(&mass[b], m);
      }
    }
    sum = smp_wave_sum(sum);
    if (lane == 0) out.block[j * 8 + wave] = sum;
  }
  if (!ask.filtered) return;
  __syncthreads();
  for (int b = tid; b < SMP_BINS; b += 512) { out.count[b] = count[b]; out.mass[b] = mass[b]; }
}

template <bool BF16>
__global__ __launch_bounds__(512) void k_sample_cut(SampleArgs a) {
  __shared__ double powers[256];
  __shared__ smp_u64 mass[SMP_BINS];
  __shared__ uint32_t count[SMP_BINS], before[SMP_BLOCKS];
  __shared__ SampleRow cut;
  __shared__ uint32_t list_at;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, s = blockIdx.y, chunk = blockIdx.x;
  const SmpAsk ask(a, s);
  if (!ask.filtered) return;
  const SampleChunk* of_row = a.chunk + static_cast<size_t>(s) * a.chunks;
  const uint32_t top = smp_row_top(a, s);
  if (top == 0) return;
  uint32_t key[4][4];
  smp_load<BF16>(a, s, chunk, key);
  if (tid >= 256) powers[tid - 256] = SMP_POWERS.v[tid - 256];
  const double per = SmpScale::per_logit(ask.T);
  const SmpScale sc(per, top);
  // the row's bins
  if (tid < SMP_BINS) {
    smp_u64 m = 0;
    uint32_t n = 0;
    for (int c = 0; c < a.chunks; ++c) {
      if (of_row[c].top == 0) continue;
      const SmpScale cs(per, of_row[c].top);
      const int db = sc.bin_shift(cs), da = sc.unit_shift(cs);
      if (tid < SMP_BINS - 1) {
        if (tid >= db) {
          n += of_row[c].count[tid - db];
          if (da < 64) m += of_row[c].mass[tid - db] >> da;
        }
      } else {
        for (int b = max(0, SMP_BINS - 1 - db); b < SMP_BINS; ++b) n += of_row[c].count[b];
      }
    }
    count[tid] = n;
    mass[tid] = m;
  }
  __syncthreads();
  if (wave == 0) {                               // bins 3 lane .. 3 lane + 2: sums up to them, and the bins that the cuts fall into
    smp_u64 n[3], m[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      n[i] = count[lane * 3 + i] + (i ? n[i - 1] : 0);
      m[i] = mass[lane * 3 + i] + (i ? m[i - 1] : 0);
    }
    const smp_u64 n0 = smp_wave_upto(n[2]) - n[2], m0 = smp_wave_upto(m[2]) - m[2];
#pragma unroll
    for (int i = 0; i < 3; ++i) { n[i] += n0; m[i] += m0; }
    auto first = [&](auto&& reached) {           // first bin with reached(sums up to it), SMP_BINS - 1 if none
      int mine = SMP_BINS - 1;
#pragma unroll
      for (int i = 2; i >= 0; --i)
        if (reached(n[i], m[i])) mine = min(mine, lane * 3 + i);
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) mine = min(mine, __shfl_xor(mine, d));
      return mine;
    };
    auto at = [&](const smp_u64 (&v)[3], int bin) {        // sum over the bins before `bin`
      if (bin <= 0) return smp_u64(0);
      const int b = bin - 1, l = b / 3, i = b - l * 3;
      const smp_u64 mine = i == 0 ? v[0] : i == 1 ? v[1] : v[2];
      return static_cast<smp_u64>(__shfl(mine, l));
    };
    SampleRow r{};
    const smp_u64 all = __shfl(m[2], 63);
    r.k_bin = SMP_BINS;
    smp_u64 least = all, most = all;             // weight that top-k leaves
    if (ask.k > 0) {
      r.k_bin = first([&](smp_u64 cn, smp_u64) { return cn >= static_cast<smp_u64>(ask.k); });
      if (r.k_bin == SMP_BINS - 1) r.k_bin = SMP_BINS;     // what is beyond weighs nothing
      else {
        r.k_above = at(n, r.k_bin);
        r.k_mass = least = at(m, r.k_bin);
        most = at(m, r.k_bin + 1);
      }
    }
    r.p_lo = SMP_BINS;
    r.p_hi = -1;
    if (ask.p < 1.f) {
      const double lo = double(ask.p) * double(least), hi = double(ask.p) * double(most);
      r.p_lo = first([&](smp_u64, smp_u64 cm) { return double(cm) >= lo && cm > 0; });
      r.p_hi = first([&](smp_u64, smp_u64 cm) { return double(cm) >= hi && cm > 0; });
      if (r.k_bin < SMP_BINS) { r.p_lo = min(r.p_lo, r.k_bin); r.p_hi = min(r.p_hi, r.k_bin); }
      r.p_mass = at(m, r.p_lo);
    }
    // elements of the cuts' bins: in the row, and in the chunks ahead of this one
    uint32_t listed = 0;
    for (int i = 0; i < 3; ++i) {
      const int b = lane * 3 + i;
      if (b == r.k_bin || (b >= r.p_lo && b <= r.p_hi)) listed += count[b];
    }
    uint32_t ahead = 0;
    for (int c = lane; c < chunk; c += 64) {
      if (of_row[c].top == 0) continue;
      const int db = sc.bin_shift(SmpScale(per, of_row[c].top));
      for (int b = r.p_lo; b <= r.p_hi; ++b)
        if (b != r.k_bin && b >= db) ahead += of_row[c].count[b - db];
      if (r.k_bin < SMP_BINS && r.k_bin >= db) ahead += of_row[c].count[r.k_bin - db];
    }
    listed = uint32_t(smp_wave_sum(listed));
    ahead = uint32_t(smp_wave_sum(ahead));
    r.listed = int(listed);
    if (lane == 0) {
      cut = r;
      list_at = ahead;
      if (chunk == 0) a.row[s] = r;
    }
  }
  __syncthreads();
  const int k_bin = cut.k_bin, p_lo = cut.p_lo, p_hi = cut.p_hi, sure = min(k_bin, p_lo);
  const bool listing = cut.listed <= SMP_LIST;
  const double floor_t = ask.least > 0.f ? log2(double(ask.least)) : -INFINITY;
  uint32_t mine[4];                              // bits of the elements to be listed
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    smp_u64 sum = 0;
    mine[j] = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (key[j][e] == 0) continue;
      const int b = sc.bin(key[j][e]);
      if (b < sure) {
        if (sc.below(key[j][e]) >= floor_t) sum += sc.mass(key[j][e], powers);
      } else if (b == k_bin || (b >= p_lo && b <= p_hi)) {
        mine[j] |= 1u << e;
      }
    }
    if (__any(sum != 0)) sum = smp_wave_sum(sum);
    if (lane == 0) a.kept[(static_cast<size_t>(s) * a.chunks + chunk) * SMP_BLOCKS + j * 8 + wave] = sum;
    const uint32_t n = uint32_t(__popcll(__ballot(mine[j] & 1)) + __popcll(__ballot(mine[j] & 2)) + __popcll(__ballot(mine[j] & 4)) + __popcll(__ballot(mine[j] & 8)));
    if (lane == 0) before[j * 8 + wave] = n;
  }
  if (!listing) return;
  __syncthreads();
  uint32_t* list = a.list + static_cast<size_t>(s) * SMP_LIST;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (!__any(mine[j] != 0)) continue;
    uint32_t at = list_at;
    for (int b = 0; b < j * 8 + wave; ++b) at += before[b];
    at += uint32_t(smp_wave_upto(__popc(mine[j]))) - __popc(mine[j]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if ((mine[j] >> e & 1) && at < SMP_LIST) list[at++] = uint32_t(chunk * SMP_CHUNK + j * 2048 + tid * 4 + e);
  }
}

// Sum over the work-group of 1024, and inclusive sums.
struct SmpGroup {
  smp_u64* part;                                 // [16]
  __device__ smp_u64 sum(smp_u64 v) const {
    v = smp_wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) v += part[w];
    return v;
  }
  __device__ smp_u64 upto(smp_u64 v) const {
    v = smp_wave_upto(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 0; w < int(threadIdx.x >> 6); ++w) v += part[w];
    return v;
  }
};

template <bool BF16>
__global__ __launch_bounds__(1024) void k_sample_draw(SampleArgs a) {
  constexpr int EACH = SMP_LIST / 1024, KEYS = 1024;
  __shared__ double powers[256];
  __shared__ smp_u64 part[16], hist[KEYS], blocks[(1 << 20) / SMP_NEIGHBOURS];
  __shared__ smp_u64 found[2];
  __shared__ int found_at;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, s = blockIdx.x, V = a.V;
  const SmpGroup group{part};
  const SmpAsk ask(a, s);
  const SampleChunk* of_row = a.chunk + static_cast<size_t>(s) * a.chunks;
  const uint32_t top = smp_row_top(a, s);
  if (top == 0) {
    if (tid == 0) {
      a.tokens[s] = -1;
      if (a.logprobs) a.logprobs[s] = -INFINITY;
    }
    return;
  }
  if (ask.greedy) {
    if (wave != 0) return;
    uint32_t first = ~0u;
    for (int c = lane; c < a.chunks; c += 64)
      if (of_row[c].top == top) first = min(first, of_row[c].top_at);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) first = min(first, uint32_t(__shfl_xor(int(first), d)));
    if (lane == 0) {
      a.tokens[s] = int(first);
      if (a.logprobs) a.logprobs[s] = 0.f;
    }
    return;
  }
  if (tid < 256) powers[tid] = SMP_POWERS.v[tid];
  const double per = SmpScale::per_logit(ask.T);
  const SmpScale sc(per, top);
  const int n_blocks = a.chunks * SMP_BLOCKS;
  const double floor_t = ask.least > 0.f ? log2(double(ask.least)) : -INFINITY;
  for (int b = tid; b < n_blocks; b += 1024) {
    if (ask.filtered) {
      blocks[b] = a.kept[static_cast<size_t>(s) * n_blocks + b];
    } else {
      const SampleChunk& c = of_row[b / SMP_BLOCKS];
      const int da = c.top ? sc.unit_shift(SmpScale(per, c.top)) : 64;
      blocks[b] = da < 64 ? c.block[b % SMP_BLOCKS] >> da : 0;
    }
  }
  __syncthreads();

  // kept: keys above `cut`, and those equal to it before index `bound`
  uint32_t cut = 0;
  int bound = V;
  if (ask.filtered) {
    const SampleRow r = a.row[s];
    const bool listing = r.listed <= SMP_LIST;
    const uint32_t* list = a.list + static_cast<size_t>(s) * SMP_LIST;
    uint32_t key[EACH], at[EACH];                // neighbours in the list are neighbours here
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int n = tid * EACH + i;
      at[i] = listing && n < r.listed ? min(list[n], uint32_t(V - 1)) : 0;
      key[i] = listing && n < r.listed ? smp_one<BF16>(a, s, int(at[i])) : 0;
    }
    const int run = (V + 1023) / 1024;           // without a list: so many logits a thread, neighbours too
    auto each = [&](auto&& f) {                  // f(key, index) of every element of bins that are in question, by each thread in order
      if (listing) {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
          if (key[i]) f(key[i], int(at[i]));
      } else {
        for (int i = tid * run; i < min(V, (tid + 1) * run); ++i) {
          const uint32_t x = smp_one<BF16>(a, s, i);
          if (x) f(x, i);
        }
      }
    };
    // The largest key with value(keys at and above it) >= target, where value() is summed over in(key, index): *above gets what lies above it.  False, and the smallest key, if all together
    // do not reach.
    auto select = [&](auto&& in, auto&& value, smp_u64 target, uint32_t* key_out, smp_u64* above) {
      uint32_t lo = ~0u, hi = 0;
      each([&](uint32_t x, int i) {
        if (in(x, i)) { lo = min(lo, x); hi = max(hi, x); }
      });
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) {
        lo = min(lo, uint32_t(__shfl_xor(int(lo), d)));
        hi = max(hi, uint32_t(__shfl_xor(int(hi), d)));
      }
      __syncthreads();
      if (lane == 0) part[wave] = smp_u64(hi) << 32 | lo;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        lo = min(lo, uint32_t(part[w]));
        hi = max(hi, uint32_t(part[w] >> 32));
      }
      smp_u64 over = 0;
      *key_out = lo;
      if (hi < lo) return false;
      while (true) {
        const uint32_t range = hi - lo;
        const int shift = max(0, 32 - __builtin_clz(range | 1) - 10);
        __syncthreads();
        hist[tid] = 0;
        if (tid == 0) found_at = KEYS;
        __syncthreads();
        each([&](uint32_t x, int i) {
          if (x >= lo && x <= hi && in(x, i)) {
            const smp_u64 v = value(x);
            if (v) atomicAdd(&hist[(hi - x) >> shift], v);
          }
        });
        __syncthreads();
        const smp_u64 mine = hist[tid], upto = over + group.upto(mine);
        if (upto >= target && upto - mine < target) {            // one bin at most
          found_at = tid;
          found[0] = upto - mine;
        }
        __syncthreads();
        const int bin = found_at;
        if (bin == KEYS) return false;
        over = found[0];
        hi = hi - (uint32_t(bin) << shift);
        if (shift == 0) {
          *key_out = hi;
          *above = over;
          return true;
        }
        lo = max(lo, hi - ((1u << shift) - 1));
      }
    };
    // the index behind the `ties`-th element with this key that is in
    auto bound_of = [&](auto&& in, uint32_t x, smp_u64 ties) {
      smp_u64 mine = 0;
      each([&](uint32_t y, int i) { mine += y == x && in(y, i); });
      const smp_u64 upto = group.upto(mine), first = upto - mine;
      if (tid == 0) found_at = V;
      __syncthreads();
      if (first < ties && ties <= upto) {
        smp_u64 n = first;
        each([&](uint32_t y, int i) {
          if (y == x && in(y, i) && ++n == ties) found_at = i + 1;
        });
      }
      __syncthreads();
      return found_at;
    };
    smp_u64 whole = 0;                           // weight that top-k leaves
    const bool cut_k = r.k_bin < SMP_BINS, cut_p = ask.p < 1.f;
    if (cut_k) {
      auto in_bin = [&](uint32_t x, int) { return sc.bin(x) == r.k_bin; };
      const smp_u64 want = static_cast<smp_u64>(ask.k) - r.k_above;
      uint32_t x;
      smp_u64 above;
      if (select(in_bin, [](uint32_t) { return smp_u64(1); }, want, &x, &above)) {
        cut = x;
        bound = bound_of(in_bin, x, want - above);
      }
      if (cut_p) {
        smp_u64 m = 0;
        each([&](uint32_t x, int i) {
          if (sc.bin(x) == r.k_bin && (x > cut || (x == cut && i < bound))) m += sc.mass(x, powers);
        });
        whole = r.k_mass + group.sum(m);
      }
    } else if (cut_p) {
      // no cut by top-k: all of the row's weight
      smp_u64 m = 0;
      for (int c = tid; c < a.chunks; c += 1024) {
        if (of_row[c].top == 0) continue;
        const int da = sc.unit_shift(SmpScale(per, of_row[c].top));
        if (da < 64)
          for (int b = 0; b < SMP_BINS; ++b) m += of_row[c].mass[b] >> da;
      }
      whole = group.sum(m);
    }
    if (cut_p) {
      const uint32_t k_cut = cut;
      const int k_bound = bound;
      auto in = [&](uint32_t x, int i) {
        const int b = sc.bin(x);
        return b >= r.p_lo && b <= r.p_hi && (x > k_cut || (x == k_cut && i < k_bound));
      };
      const double goal = double(ask.p) * double(whole) - double(r.p_mass);
      const smp_u64 target = goal > 1. ? static_cast<smp_u64>(ceil(goal)) : 1;       // the first one is kept always
      uint32_t x;
      smp_u64 above;
      if (select(in, [&](uint32_t y) { return sc.mass(y, powers); }, target, &x, &above)) {
        const smp_u64 w = sc.mass(x, powers), ties = (target - above + w - 1) / w;
        const int b = bound_of(in, x, ties);
        cut = x;
        bound = x == k_cut ? min(b, k_bound) : b;
      } else if (x > k_cut && x != ~0u) {        // short of it by the last units: all of these bins
        cut = x;
        bound = V;
      }
    }
    // what is kept of those bins joins the sums of its neighbourhoods
    const int sure = min(r.k_bin, r.p_lo);
    each([&](uint32_t x, int i) {
      const int b = sc.bin(x);
      if (b < sure || (b != r.k_bin && (b < r.p_lo || b > r.p_hi))) return;
      if ((x > cut || (x == cut && i < bound)) && sc.below(x) >= floor_t) atomicAdd(&blocks[i / SMP_NEIGHBOURS], sc.mass(x, powers));
    });
    __syncthreads();
  }

  // the neighbourhood: thread t has blocks 4 t .. 4 t + 3
  smp_u64 mine = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) mine += tid * 4 + i < n_blocks ? blocks[tid * 4 + i] : 0;
  const smp_u64 upto = group.upto(mine);
  if (tid == 1023) found[1] = upto;
  __syncthreads();
  const smp_u64 W = found[1];
  float u = a.u[s];
  u = u > 0.f ? fminf(u, 1.f) : 0.f;
  // the first running weight above u W; in integers: of at least floor(u W) + 1, and W where u is 1
  const double goal_d = floor(double(u) * double(W));
  smp_u64 goal = static_cast<smp_u64>(goal_d) + 1;
  goal = goal > W ? W : goal;
  if (upto >= goal && upto - mine < goal) {
    smp_u64 run = upto - mine;
    int b = tid * 4;
    while (run + blocks[b] < goal) run += blocks[b++];
    found_at = b;
    found[0] = goal - run;
  }
  __syncthreads();
  if (wave != 0) return;
  const int block = found_at;
  goal = found[0];
  uint32_t x[4];
  smp_u64 m[4], own = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int i = block * SMP_NEIGHBOURS + lane * 4 + e;
    x[e] = i < V ? smp_one<BF16>(a, s, i) : 0;
    const bool in = x[e] != 0 && (x[e] > cut || (x[e] == cut && i < bound)) && sc.below(x[e]) >= floor_t;
    m[e] = in ? sc.mass(x[e], powers) : 0;
    own += m[e];
  }
  const smp_u64 run_upto = smp_wave_upto(own), in_block = __shfl(run_upto, 63);
  if (goal > in_block) goal = in_block;          // sums of a chunk's units and of the row's may differ in the last unit
  if (run_upto >= goal && run_upto - own < goal) {
    smp_u64 run = run_upto - own;
    int e = 0;
    while (e < 3 && run + m[e] < goal) run += m[e++];
    const uint32_t k = e == 0 ? x[0] : e == 1 ? x[1] : e == 2 ? x[2] : x[3];
    a.tokens[s] = block * SMP_NEIGHBOURS + lane * 4 + e;
    if (a.logprobs) {
      a.logprobs[s] = float((sc.units(k) - log2(double(W))) * 0.69314718055994530942);
    }
  }
}

namespace {
struct SampleSpace { size_t row, kept, list, total; };
SampleSpace space(int S, int V) {
  const size_t chunks = (size_t(V) + SMP_CHUNK - 1) / SMP_CHUNK;
  SampleSpace p;
  p.row = align256(size_t(S) * chunks * sizeof(SampleChunk));
  p.kept = p.row + align256(size_t(S) * sizeof(SampleRow));
  p.list = p.kept + align256(size_t(S) * chunks * SMP_BLOCKS * 8);
  p.total = p.list + align256(size_t(S) * SMP_LIST * 4);
  return p;
}
}  // namespace

size_t sample_ws_bytes(int S, int V) { return space(S, V).total; }

int32_t launch_sample(const void* logits, bool bf16, long long stride, int S, int V, const moqe_sampling& how, const float* u, int32_t* tokens, float* logprobs,
                      void* ws, hipStream_t st) {
  const SampleSpace p = space(S, V);
  uint8_t* b = static_cast<uint8_t*>(ws);
  SampleArgs a{logits, stride, how.temperature, how.top_k, how.top_p, how.min_p, u, tokens, logprobs, S, V, (V + SMP_CHUNK - 1) / SMP_CHUNK,
               reinterpret_cast<SampleChunk*>(b), reinterpret_cast<SampleRow*>(b + p.row), reinterpret_cast<smp_u64*>(b + p.kept), reinterpret_cast<uint32_t*>(b + p.list)};
  ProfileScope ps(MOQE_PK_OTHER, st);
  const bool filters = how.top_k || how.top_p || how.min_p;
  const dim3 chunks(a.chunks, S);
  auto go = [&](auto bf) {
    constexpr bool BF16 = decltype(bf)::value;
    hipLaunchKernelGGL((k_sample_chunks<BF16>), chunks, dim3(512), 0, st, a);
    if (filters) hipLaunchKernelGGL((k_sample_cut<BF16>), chunks, dim3(512), 0, st, a);
    hipLaunchKernelGGL((k_sample_draw<BF16>), dim3(S), dim3(1024), 0, st, a);
  };
  if (bf16) go(std::true_type());
  else go(std::false_type());
  return check_launch("sample");
}

}  // namespace moqe
