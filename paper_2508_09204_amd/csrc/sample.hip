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

constexpr int SMP_THREADS = 512, SMP_NEIGHBOURS = 256;
constexpr int SMP_BINS = 192;                  // quarters of an octave below the largest; the last one: everything that weighs nothing (2^-47 and less)
constexpr int SMP_LIST = 4096;                 // of a row: longer lists are read from the logits instead
constexpr int SMP_ONE = 43;

typedef unsigned long long smp_u64;

struct SampleArgs {
  const void* logits; long long stride;
  const float* temperature; const int32_t* top_k; const float *top_p, *min_p; const float* u;
  int32_t* tokens; float* logprobs;
  int32_t S, V, chunks, blocks;                // blocks: of SMP_NEIGHBOURS logits, as the chunks have them
  struct SampleChunk* chunk; struct SampleRow* row; smp_u64* block; uint32_t* list;      // [S][chunks], [S], [S][blocks], [S][SMP_LIST]
};
struct SampleChunk {
  uint32_t top, top_at;                        // largest key and its first index; 0: nothing but minus infinity and NaN
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

// A thread's logits as keys: four at each of P places, SMP_NEIGHBOURS to a wave and place.  Past the row's end: 0.
template <bool BF16, int P>
__device__ __forceinline__ void smp_load(const SampleArgs& a, int s, int chunk, uint32_t (&key)[P][4]) {
  const char* row = static_cast<const char*>(a.logits) + s * a.stride * (BF16 ? 2 : 4);
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const int i = (chunk * P + j) * (SMP_THREADS * 4) + int(threadIdx.x) * 4;
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

// Sums and maxima over a wave by moves between lanes in registers: rows of 16, then across them.  Lanes that get nothing get 0.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t smp_move(uint32_t v) { return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, ROWS, 0xf, false)); }
template <int CTRL, int ROWS>
__device__ __forceinline__ smp_u64 smp_move(smp_u64 v) { return smp_u64(smp_move<CTRL, ROWS>(uint32_t(v >> 32))) << 32 | smp_move<CTRL, ROWS>(uint32_t(v)); }
template <typename T, typename F>
__device__ __forceinline__ T smp_upto(T v, F&& f) {
  v = f(v, smp_move<0x111, 0xf>(v));           // row_shr:1, 2, 4, 8
  v = f(v, smp_move<0x112, 0xf>(v));
  v = f(v, smp_move<0x114, 0xf>(v));
  v = f(v, smp_move<0x118, 0xf>(v));
  v = f(v, smp_move<0x142, 0xa>(v));           // row_bcast:15, row_bcast:31
  return f(v, smp_move<0x143, 0xc>(v));
}
__device__ __forceinline__ uint32_t smp_lane(uint32_t v, int lane) { return uint32_t(__builtin_amdgcn_readlane(int(v), lane)); }
__device__ __forceinline__ smp_u64 smp_lane(smp_u64 v, int lane) { return smp_u64(smp_lane(uint32_t(v >> 32), lane)) << 32 | smp_lane(uint32_t(v), lane); }
template <typename T> __device__ __forceinline__ T smp_wave_upto(T v) { return smp_upto(v, [](T a, T b) { return a + b; }); }       // inclusive
template <typename T> __device__ __forceinline__ T smp_wave_sum(T v) { return smp_lane(smp_wave_upto(v), 63); }
__device__ __forceinline__ uint32_t smp_wave_max(uint32_t v) { return smp_lane(smp_upto(v, [](uint32_t a, uint32_t b) { return max(a, b); }), 63); }

// What is asked of a row.
struct SmpAsk {
  float T, p, least;
  int k;                             // 0: all
  bool greedy, filtered;
  __device__ SmpAsk(const SampleArgs& a, int s) {
    // all four asked for at once
    const float t = (a.temperature ? a.temperature : a.u)[s], q = (a.top_p ? a.top_p : a.u)[s], m = (a.min_p ? a.min_p : a.u)[s];
    const int n = (a.top_k ? a.top_k : reinterpret_cast<const int32_t*>(a.u))[s];
    T = a.temperature ? t : 1.f;
    greedy = !(T > 0.f);
    k = a.top_k && n >= 1 && n < a.V ? n : 0;
    p = a.top_p && q < 1.f ? q : 1.f;
    if (!(p > 0.f)) p = 0.f;
    least = a.min_p && m > 0.f ? fminf(m, 1.f) : 0.f;
    filtered = !greedy && (k > 0 || p < 1.f || least > 0.f);
  }
};

// Largest key of the row, by all lanes of a wave.
__device__ __forceinline__ uint32_t smp_row_top(const SampleArgs& a, int s) {
  uint32_t top = 0;
  for (int c = threadIdx.x & 63; c < a.chunks; c += 64) top = max(top, a.chunk[static_cast<size_t>(s) * a.chunks + c].top);
  return smp_wave_max(top);
}

template <bool BF16, int P>
__global__ __launch_bounds__(SMP_THREADS) void k_sample_chunks(SampleArgs a) {
  __shared__ double powers[256];
  __shared__ uint32_t tops[8], count[SMP_BINS];
  __shared__ smp_u64 mass[SMP_BINS];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, s = blockIdx.y, chunk = blockIdx.x;
  SampleChunk& out = a.chunk[static_cast<size_t>(s) * a.chunks + chunk];
  uint32_t key[P][4];
  smp_load<BF16, P>(a, s, chunk, key);
  if (tid < 256) powers[tid] = SMP_POWERS.v[tid];
  const SmpAsk ask(a, s);
  if (tid < SMP_BINS) { count[tid] = 0; mass[tid] = 0; }
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < P; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, key[j][e]);
  top = smp_wave_max(top);
  if (lane == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) top = max(top, tops[w]);
  if (ask.greedy) {                            // the first index of the largest
    uint32_t first = ~0u;
#pragma unroll
    for (int j = P - 1; j >= 0; --j)
#pragma unroll
      for (int e = 3; e >= 0; --e)
        if (key[j][e] == top) first = uint32_t((chunk * P + j) * (SMP_THREADS * 4) + tid * 4 + e);
    first = ~smp_wave_max(~first);
    __syncthreads();
    if (lane == 0) tops[wave] = first;
    __syncthreads();
    if (tid == 0) {
#pragma unroll
      for (int w = 0; w < 8; ++w) first = min(first, tops[w]);
      out.top = top;
      out.top_at = first;
    }
    return;
  }
  if (tid == 0) out.top = top;
  if (top == 0) return;
  const SmpScale sc(SmpScale::per_logit(ask.T), top);
  const bool bins = ask.k > 0 || ask.p < 1.f;
  smp_u64* block = a.block + static_cast<size_t>(s) * a.blocks + chunk * (P * 8) + wave;
#pragma unroll
  for (int j = 0; j < P; ++j) {
    smp_u64 sum = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const smp_u64 m = !ask.filtered || ask.p < 1.f ? sc.mass(key[j][e], powers) : 0;
      sum += m;
      if (bins && key[j][e] != 0) {
        const int b = sc.bin(key[j][e]);
        atomicAdd(&count[b], 1u);
        if (ask.p < 1.f && m) atomicAdd(&mass[b], m);
      }
    }
    if (!ask.filtered) {
      sum = smp_wave_sum(sum);
      if (lane == 0) block[j * 8] = sum;
    }
  }
  if (!bins) return;
  __syncthreads();
  if (tid < SMP_BINS) { out.count[tid] = count[tid]; out.mass[tid] = mass[tid]; }
}

constexpr int SMP_CHUNKS = 128;                  // of a row at most

template <bool BF16, int P>
__global__ __launch_bounds__(SMP_THREADS) void k_sample_cut(SampleArgs a) {
  constexpr int BLOCKS = P * 8;
  __shared__ double powers[256];
  __shared__ smp_u64 mass[2][SMP_BINS];
  __shared__ uint32_t count[2][SMP_BINS], before[BLOCKS];
  __shared__ int bins_down[SMP_CHUNKS], units_down[SMP_CHUNKS];
  __shared__ SampleRow cut;
  __shared__ uint32_t list_at;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, s = blockIdx.y, chunk = blockIdx.x;
  const SmpAsk ask(a, s);
  if (!ask.filtered) return;
  const SampleChunk* of_row = a.chunk + static_cast<size_t>(s) * a.chunks;
  uint32_t key[P][4];
  smp_load<BF16, P>(a, s, chunk, key);
  if (tid >= 256) powers[tid - 256] = SMP_POWERS.v[tid - 256];
  const uint32_t top = smp_row_top(a, s);
  if (top == 0) return;
  const double per = SmpScale::per_logit(ask.T);
  const SmpScale sc(per, top);
  const bool bins = ask.k > 0 || ask.p < 1.f;
  if (tid < a.chunks) {
    const uint32_t t = of_row[tid].top;
    const SmpScale cs(per, t ? t : 1);
    bins_down[tid] = t ? sc.bin_shift(cs) : SMP_BINS;
    units_down[tid] = t ? sc.unit_shift(cs) : 64;
  }
  __syncthreads();
  if (bins && tid < 2 * SMP_BINS) {              // the row's bins, half the chunks each; what lies past the last one weighs nothing and is not counted
    const int half = tid / SMP_BINS, b = tid - half * SMP_BINS, end = (half + 1) * a.chunks / 2;
    smp_u64 m = 0;
    uint32_t n = 0;
#pragma unroll 8
    for (int c = half * a.chunks / 2; c < end; ++c) {
      const int db = bins_down[c], da = units_down[c], from = b - db;
      if (from >= 0) {
        n += of_row[c].count[from];
        if (da < 64) m += of_row[c].mass[from] >> da;
      }
    }
    count[half][b] = n;
    mass[half][b] = m;
  }
  __syncthreads();
  if (wave == 0) {
    SampleRow r{};
    r.k_bin = r.p_lo = SMP_BINS;
    r.p_hi = -1;
    uint32_t ahead = 0;
    if (bins) {                                  // bins 3 lane .. 3 lane + 2: sums up to them, and the bins that the cuts fall into
      smp_u64 n[3], m[3];
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        n[i] = count[0][lane * 3 + i] + count[1][lane * 3 + i] + (i ? n[i - 1] : 0);
        m[i] = mass[0][lane * 3 + i] + mass[1][lane * 3 + i] + (i ? m[i - 1] : 0);
      }
      const uint32_t in_bin[3] = {uint32_t(n[0]), uint32_t(n[1] - n[0]), uint32_t(n[2] - n[1])};
      const smp_u64 n0 = smp_wave_upto(n[2]) - n[2], m0 = smp_wave_upto(m[2]) - m[2];
#pragma unroll
      for (int i = 0; i < 3; ++i) { n[i] += n0; m[i] += m0; }
      auto first = [&](auto&& reached) {         // first bin with reached(sums up to it), which holds for all after it; SMP_BINS - 1 if none
        const int mine = reached(n[0], m[0]) ? 0 : reached(n[1], m[1]) ? 1 : 2;
        const smp_u64 hit = __ballot(reached(n[2], m[2]));
        if (hit == 0) return SMP_BINS - 1;
        const int l = __builtin_ctzll(hit);
        return l * 3 + __builtin_amdgcn_readlane(mine, l);
      };
      auto before_bin = [&](const smp_u64 (&v)[3], int bin) {        // sum over the bins before it
        if (bin <= 0) return smp_u64(0);
        const int b = bin - 1, l = b / 3, i = b - l * 3;
        return i == 0 ? smp_lane(v[0], l) : i == 1 ? smp_lane(v[1], l) : smp_lane(v[2], l);
      };
      const smp_u64 all = smp_lane(m[2], 63);
      smp_u64 least = all, most = all;           // weight that top-k leaves
      if (ask.k > 0) {
        r.k_bin = first([&](smp_u64 cn, smp_u64) { return cn >= static_cast<smp_u64>(ask.k); });
        if (r.k_bin == SMP_BINS - 1) r.k_bin = SMP_BINS;     // what is beyond weighs nothing
        else {
          r.k_above = before_bin(n, r.k_bin);
          r.k_mass = least = before_bin(m, r.k_bin);
          most = before_bin(m, r.k_bin + 1);
        }
      }
      if (r.k_bin == SMP_BINS) r.k_mass = all;
      if (ask.p < 1.f) {
        const double lo = double(ask.p) * double(least), hi = double(ask.p) * double(most);
        r.p_lo = first([&](smp_u64, smp_u64 cm) { return double(cm) >= lo && cm > 0; });
        r.p_hi = first([&](smp_u64, smp_u64 cm) { return double(cm) >= hi && cm > 0; });
        if (r.k_bin < SMP_BINS) { r.p_lo = min(r.p_lo, r.k_bin); r.p_hi = min(r.p_hi, r.k_bin); }
        r.p_mass = before_bin(m, r.p_lo);
      }
      // elements of the cuts' bins: in the row, and in the chunks ahead of this one
      uint32_t listed = 0;
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const int b = lane * 3 + i;
        if (b == r.k_bin || (b >= r.p_lo && b <= r.p_hi)) listed += in_bin[i];
      }
      r.listed = int(smp_wave_sum(listed));
      for (int c = lane; c < chunk; c += 64) {
        const int db = bins_down[c];
        for (int b = max(r.p_lo, db); b <= r.p_hi; ++b)
          if (b != r.k_bin) ahead += of_row[c].count[b - db];
        if (r.k_bin < SMP_BINS && r.k_bin >= db) ahead += of_row[c].count[r.k_bin - db];
      }
      ahead = smp_wave_sum(ahead);
    }
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
  smp_u64* block = a.block + static_cast<size_t>(s) * a.blocks + chunk * BLOCKS + wave;
  uint32_t mine[P];                              // bits of the elements to be listed
#pragma unroll
  for (int j = 0; j < P; ++j) {
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
    if (lane == 0) block[j * 8] = sum;
    const uint32_t n = uint32_t(__popcll(__ballot(mine[j] & 1)) + __popcll(__ballot(mine[j] & 2)) + __popcll(__ballot(mine[j] & 4)) + __popcll(__ballot(mine[j] & 8)));
    if (lane == 0) before[j * 8 + wave] = n;
  }
  if (!bins || !listing) return;
  __syncthreads();
  uint32_t* list = a.list + static_cast<size_t>(s) * SMP_LIST;
  const uint32_t ahead_of = smp_wave_upto(lane < BLOCKS ? before[lane] : 0u);
#pragma unroll
  for (int j = 0; j < P; ++j) {
    if (!__any(mine[j] != 0)) continue;
    const int b = __builtin_amdgcn_readfirstlane(j * 8 + wave);
    uint32_t at = list_at + (b ? smp_lane(ahead_of, b - 1) : 0u) + smp_wave_upto(uint32_t(__popc(mine[j]))) - __popc(mine[j]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if ((mine[j] >> e & 1) && at < SMP_LIST) list[at++] = uint32_t((chunk * P + j) * (SMP_THREADS * 4) + tid * 4 + e);
  }
}

// Sum over the work-group, and inclusive sums.
struct SmpGroup {
  smp_u64* part;                                 // [8]
  __device__ smp_u64 sum(smp_u64 v) const {
    v = smp_wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) v += part[w];
    return v;
  }
  __device__ smp_u64 upto(smp_u64 v) const {
    v = smp_wave_upto(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 7; ++w) v += w < int(threadIdx.x >> 6) ? part[w] : 0;
    return v;
  }
};

template <bool BF16>
__global__ __launch_bounds__(SMP_THREADS) void k_sample_draw(SampleArgs a) {
  constexpr int EACH = SMP_LIST / SMP_THREADS, KEYS = 1024, PER = (1 << 20) / SMP_NEIGHBOURS / SMP_THREADS;
  __shared__ double powers[256];
  __shared__ smp_u64 part[8], hist[KEYS], blocks[(1 << 20) / SMP_NEIGHBOURS];
  __shared__ smp_u64 found[2];
  __shared__ int found_at, units_down[SMP_CHUNKS];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, s = blockIdx.x, V = a.V;
  const SmpGroup group{part};
  const SmpAsk ask(a, s);
  const SampleChunk* of_row = a.chunk + static_cast<size_t>(s) * a.chunks;
  const int n_blocks = a.blocks, per_chunk = n_blocks / a.chunks;
  const smp_u64* row_blocks = a.block + static_cast<size_t>(s) * n_blocks;
  smp_u64 first_blocks = tid < n_blocks ? row_blocks[tid] : 0;        // asked for before it is known how they count
  if (tid < 256) powers[tid] = SMP_POWERS.v[tid];
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
    first = ~smp_wave_max(~first);
    if (lane == 0) {
      a.tokens[s] = int(first);
      if (a.logprobs) a.logprobs[s] = 0.f;
    }
    return;
  }
  const double per = SmpScale::per_logit(ask.T);
  const SmpScale sc(per, top);
  const double floor_t = ask.least > 0.f ? log2(double(ask.least)) : -INFINITY;
  if (tid < a.chunks) {
    const uint32_t t = of_row[tid].top;
    units_down[tid] = t ? ask.filtered ? 0 : sc.unit_shift(SmpScale(per, t)) : 64;
  }
  __syncthreads();
  for (int b = tid; b < n_blocks; b += SMP_THREADS) {
    const int da = units_down[b / per_chunk];
    const smp_u64 v = b == tid ? first_blocks : row_blocks[b];
    blocks[b] = da < 64 ? v >> da : 0;
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
    const int run = (V + SMP_THREADS - 1) / SMP_THREADS;           // without a list: so many logits a thread, neighbours too
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
      lo = ~smp_wave_max(~lo);
      hi = smp_wave_max(hi);
      __syncthreads();
      if (lane == 0) part[wave] = smp_u64(hi) << 32 | lo;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < 8; ++w) {
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
        hist[2 * tid] = hist[2 * tid + 1] = 0;
        if (tid == 0) found_at = KEYS;
        __syncthreads();
        each([&](uint32_t x, int i) {
          if (x >= lo && x <= hi && in(x, i)) {
            const smp_u64 v = value(x);
            if (v) atomicAdd(&hist[(hi - x) >> shift], v);
          }
        });
        __syncthreads();
        const smp_u64 one = hist[2 * tid], two = hist[2 * tid + 1], upto = over + group.upto(one + two), ahead = upto - one - two;
        if (upto >= target && ahead < target) {                  // one thread at most
          const bool second = ahead + one < target;
          found_at = 2 * tid + second;
          found[0] = ahead + (second ? one : 0);
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
      whole = r.k_mass;                          // no cut by top-k: all of the row's weight
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

  // the neighbourhood: thread t has some that follow one another
  const int each_t = (n_blocks + SMP_THREADS - 1) / SMP_THREADS, b0 = tid * each_t, b1 = min(n_blocks, b0 + each_t);
  static_assert(PER <= 8, "");
  smp_u64 mine = 0;
  for (int b = b0; b < b1; ++b) mine += blocks[b];
  const smp_u64 upto = group.upto(mine);
  if (tid == SMP_THREADS - 1) found[1] = upto;
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
    int b = b0;
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
  const smp_u64 run_upto = smp_wave_upto(own), in_block = smp_lane(run_upto, 63);
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
struct SampleSpace { int places, chunks; size_t row, block, list, total; };
SampleSpace space(int S, int V) {
  SampleSpace p;
  p.places = static_cast<long long>(S) * V < (1 << 21) && V <= SMP_CHUNKS * SMP_THREADS * 4 ? 1 : 4;
  p.chunks = (V + p.places * SMP_THREADS * 4 - 1) / (p.places * SMP_THREADS * 4);
  p.row = align256(size_t(S) * p.chunks * sizeof(SampleChunk));
  p.block = p.row + align256(size_t(S) * sizeof(SampleRow));
  p.list = p.block + align256(size_t(S) * p.chunks * p.places * 8 * 8);
  p.total = p.list + align256(size_t(S) * SMP_LIST * 4);
  return p;
}
}  // namespace

size_t sample_ws_bytes(int S, int V) { return space(S, V).total; }

int32_t launch_sample(const void* logits, bool bf16, long long stride, int S, int V, const moqe_sampling& how, const float* u, int32_t* tokens, float* logprobs,
                      void* ws, hipStream_t st) {
  const SampleSpace p = space(S, V);
  uint8_t* b = static_cast<uint8_t*>(ws);
  SampleArgs a{logits, stride, how.temperature, how.top_k, how.top_p, how.min_p, u, tokens, logprobs, S, V, p.chunks, p.chunks * p.places * 8,
               reinterpret_cast<SampleChunk*>(b), reinterpret_cast<SampleRow*>(b + p.row), reinterpret_cast<smp_u64*>(b + p.block), reinterpret_cast<uint32_t*>(b + p.list)};
  ProfileScope ps(MOQE_PK_OTHER, st);
  const bool filters = how.top_k || how.top_p || how.min_p;
  const dim3 chunks(p.chunks, S), threads(SMP_THREADS);
  auto go = [&](auto bf, auto places) {
    constexpr bool BF16 = decltype(bf)::value;
    constexpr int P = decltype(places)::value;
    hipLaunchKernelGGL((k_sample_chunks<BF16, P>), chunks, threads, 0, st, a);
    if (filters) hipLaunchKernelGGL((k_sample_cut<BF16, P>), chunks, threads, 0, st, a);
    hipLaunchKernelGGL((k_sample_draw<BF16>), dim3(S), threads, 0, st, a);
  };
  auto with = [&](auto bf) {
    if (p.places == 1) go(bf, std::integral_constant<int, 1>());
    else go(bf, std::integral_constant<int, 4>());
  };
  if (bf16) with(std::true_type());
  else with(std::false_type());
  return check_launch("sample");
}

}  // namespace moqe
