// Tokens from logits by temperature, top-k, top-p and min-p.
//
// Weights are 2^t for t = l log2(e) / T, and everything that decides is an integer sum, from a table of 2^(j / 256) and a cubic (2^-42 of a weight).  A weight is counted in 2^-43 of the power of
// two above the largest weight of what it is summed with first, which no division of a row over work-groups changes: a bin (a quarter of an octave) for the cuts, 256 neighbours for the draw
// of rows without filters, the whole row where its largest is known.  Sums of different units differ by a shift, on the sum.  So neither a row's division nor the order of atomics changes a result.
//
//   k_sample_chunks  2048 or 8192 logits a work-group: their largest, sums of 256 neighbours, and (rows with cuts) counts and weights of bins a quarter of an octave wide, counted down from
//                    the largest
//   k_sample_cut     filtered rows, again by chunks: the bins of the whole row give those that the cuts of top-k and top-p fall into; sums of 256 neighbours that are kept for sure, and a list
//                    of what lies in the cuts' bins
//   k_sample_draw    a work-group a row: the cuts inside their bins, by counting keys in 1024 bins, then in 1024 of the one they fall into, until a bin is one key; the neighbourhood that the
//                    running weight passes u W in; the token in it
// The logits are read once from memory, and a second time, from the caches, where there are filters.
// 256 rows of 32000 without cuts 19.0 us: 64-bit arithmetic of a table and a cubic a logit (17.0 with units of a whole chunk, in which an element can weigh nothing where its neighbourhood does not);
// 64 rows of 128000 with cuts 57 (18 chunks, 25 cut, 18 draw under the profiler), one row of 32000 22 (4, 7 and 12): launches and trips to memory that wait for one another.
#include "moqe_internal.h"

#include <type_traits>

namespace moqe {

constexpr int SMP_THREADS = 512, SMP_NEIGHBOURS = 256;
constexpr int SMP_CHUNKS = 128;                // of a row at most
constexpr int SMP_BLOCKS = (1 << 20) / SMP_NEIGHBOURS;      // neighbourhoods of a row at most
constexpr int SMP_BINS = 192;                  // quarters of an octave below the largest; the last one: everything that weighs nothing (2^-47 and less)
constexpr int SMP_COPIES = 4;                  // of the bins while they are counted, for neighbouring lanes: most logits of a wave fall into a few
constexpr int SMP_LIST = 16384;                // of a row at most: where the cuts' bins have more, the row is read instead
constexpr int SMP_HELD = 4096;                 // of them in LDS: longer lists are read again for every pass
constexpr int SMP_ONE = 43;

typedef unsigned long long smp_u64;

struct SampleArgs {
  const void* logits; long long stride;
  const float* temperature; const int32_t* top_k; const float *top_p, *min_p; const float* u;
  int32_t* tokens; float* logprobs;
  int32_t S, V, chunks, blocks, list_size;     // blocks: of SMP_NEIGHBOURS logits, as the chunks have them
  struct SampleChunk* chunk; struct SampleRow* row; smp_u64* block; float* block_top; uint2* list;      // [S][chunks], [S], [S][blocks] twice, [S][list_size] (bits, index)
};
struct SampleChunk {
  float top;                                   // minus infinity: there is nothing else
  uint32_t top_at;                             // first index of the largest (rows of temperature 0)
  smp_u64 mass[SMP_BINS];                      // in units of the bin (rows cut by top-p)
  uint32_t count[SMP_BINS];
};
struct SampleRow {                             // where the cuts lie
  int32_t k_bin, p_lo, p_hi, listed;           // bin of the cut of top-k (SMP_BINS: none), first and last bin that the cut of top-p may lie in (none: SMP_BINS, -1), elements of those bins
  smp_u64 k_above, k_mass, p_mass;             // elements above k_bin, weight above it, weight above p_lo
};

// A finite value as an integer of the same order; of bf16 values the upper half says it all.
template <bool BF16>
__device__ __forceinline__ uint32_t smp_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f), k = (b >> 31) ? ~b : b | 0x80000000u;                // -0 as +0
  return BF16 ? k >> 16 : k;
}
template <bool BF16>
__device__ __forceinline__ float smp_value(uint32_t key) {
  const uint32_t k = BF16 ? key << 16 | ((key >> 15) ? 0u : 0xffffu) : key;
  return __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k);
}

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

// How logits weigh, given the largest (of 256 neighbours, of a chunk, of the row).  Differences of logits come first: they are exact or nearly so, also where t itself is far from 0.  Of a largest
// of plus infinity the others count as minus infinity and the infinite ones as 0 (clean()).
struct SmpScale {
  double c, c256, top_v, top_t, octave, shift, floor4;
  bool infinite;
  static __device__ double per_logit(float T) { return T > 0.f ? 1.4426950408889634074 / double(T) : 0.0; }
  __device__ SmpScale(double c_, float top) : c(c_), c256(c_ * 256), infinite(top == INFINITY) {
    top_v = infinite ? 0.0 : double(top);
    top_t = top_v * c;
    octave = floor(top_t);
    const double part = top_t - octave;
    shift = (part + lost(top_v, top_t) + (SMP_ONE - 1)) * 256;
    floor4 = floor(top_t * 4);
  }
  // What the rounded product t = v c lacks.  Where t has no digits behind the point (T is tiny), logits that differ are octaves apart and it does not matter.
  __device__ double lost(double v, double t) const { return fabs(t) < 4503599627370496.0 ? fma(v, c, -t) : 0.0; }
  __device__ float clean(float v) const { return infinite ? (v == INFINITY ? 0.f : -INFINITY) : v; }
  // how many units of the other (of some of the row's logits) are one of this (the row's), as a shift; bins between their largest
  __device__ int unit_shift(const SmpScale& other) const {
    if (infinite != other.infinite) return 64;
    const double d = octave - other.octave;
    return d < 64 ? int(d) : 64;
  }
  __device__ int bin_shift(const SmpScale& chunk) const {
    if (infinite != chunk.infinite) return SMP_BINS;
    const double d = floor4 - chunk.floor4;
    return d < SMP_BINS ? int(d) : SMP_BINS;
  }
  __device__ int bin_unit_shift(int bin) const { return int(octave - floor((floor4 - bin) * 0.25)); }       // as unit_shift(), for a bin's units
  __device__ int bin(float v) const { return int(fmin(floor4 - floor(double(v) * c * 4), double(SMP_BINS - 1))); }
  __device__ double below(float v) const { return (double(v) - top_v) * c; }           // log2 of its weight over the largest
  // 2^(u / 256), u at least -512, to an integer in the last bits of a double of 2^52 and more.  0 from 2^-2 on.
  static __device__ double power_bits(double u, const double* powers) {
    const double magic = 6755399441055744.0, n = u + magic, r = u - (n - magic);       // 1.5 * 2^52: the integer next to u stands in the last bits
    const int i = int(uint32_t(__builtin_bit_cast(smp_u64, n)));
    constexpr double L = 0.69314718055994530942 / 256;
    const double p = fma(r, fma(r, fma(r, L * L * L / 6, L * L / 2), L), 1.0) * powers[i & 255];
    return __builtin_bit_cast(double, __builtin_bit_cast(smp_u64, p) + (smp_u64(uint32_t(i & ~255) << 12) << 32)) + 4503599627370496.0;      // times 2^(i / 256), plus 2^52
  }
  // Its weight in units.  Minus infinity weighs nothing.
  __device__ double mass_bits(float v, const double* powers) const { return power_bits(fmax(fma(double(v) - top_v, c256, shift), -512.0), powers); }
  __device__ smp_u64 mass(float v, const double* powers) const { return __builtin_bit_cast(smp_u64, mass_bits(v, powers)) & 0xfffffffffffffull; }
  // Its weight in units of its bin, 2^-43 of the power of two above the bin: a matter of the logit alone.
  __device__ smp_u64 bin_mass(float v, const double* powers) const {
    const double t = double(v) * c, whole = floor(t), part = t - whole;
    return __builtin_bit_cast(smp_u64, power_bits((part + lost(double(v), t) + (SMP_ONE - 1)) * 256, powers)) & 0xfffffffffffffull;
  }
  __device__ double units(float v) const { return below(v) + shift * (1.0 / 256); }    // log2 of its mass
};

__device__ __forceinline__ float smp_no_nan(float v) { return v > -INFINITY ? v : -INFINITY; }

// A thread's logits: four at each of P places, SMP_NEIGHBOURS to a wave and place.  NaN, and what lies past the row's end, as minus infinity.
template <bool BF16, int P>
__device__ __forceinline__ void smp_load(const SampleArgs& a, int s, int chunk, float (&v)[P][4]) {
  const char* row = static_cast<const char*>(a.logits) + s * a.stride * (BF16 ? 2 : 4);
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const int i = (chunk * P + j) * (SMP_THREADS * 4) + int(threadIdx.x) * 4;
    if (i + 4 <= a.V) {                                         // wide loads need no alignment beyond an element's
      if constexpr (BF16) {
        uint2 w;
        __builtin_memcpy(&w, row + i * 2ll, 8);
        v[j][0] = __uint_as_float(w.x << 16); v[j][1] = __uint_as_float(w.x & 0xffff0000u); v[j][2] = __uint_as_float(w.y << 16); v[j][3] = __uint_as_float(w.y & 0xffff0000u);
      } else {
        uint4 w;
        __builtin_memcpy(&w, row + i * 4ll, 16);
        v[j][0] = __uint_as_float(w.x); v[j][1] = __uint_as_float(w.y); v[j][2] = __uint_as_float(w.z); v[j][3] = __uint_as_float(w.w);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[j][e] = -INFINITY;
        if (i + e < a.V) v[j][e] = BF16 ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(row)[i + e]) << 16) : reinterpret_cast<const float*>(row)[i + e];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < P; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[j][e] = smp_no_nan(v[j][e]);
}
template <bool BF16>
__device__ __forceinline__ float smp_one(const SampleArgs& a, int s, int i) {
  if constexpr (BF16) return smp_no_nan(__uint_as_float(uint32_t(static_cast<const uint16_t*>(a.logits)[s * a.stride + i]) << 16));
  else return smp_no_nan(static_cast<const float*>(a.logits)[s * a.stride + i]);
}

// Sums and maxima over a wave by moves between lanes in registers: rows of 16, then across them.  Lanes that get nothing get `none`.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t smp_move(uint32_t v, uint32_t none) { return uint32_t(__builtin_amdgcn_update_dpp(int(none), int(v), CTRL, ROWS, 0xf, false)); }
template <int CTRL, int ROWS>
__device__ __forceinline__ smp_u64 smp_move(smp_u64 v, smp_u64 none) {
  return smp_u64(smp_move<CTRL, ROWS>(uint32_t(v >> 32), uint32_t(none >> 32))) << 32 | smp_move<CTRL, ROWS>(uint32_t(v), uint32_t(none));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float smp_move(float v, float none) { return __uint_as_float(smp_move<CTRL, ROWS>(__float_as_uint(v), __float_as_uint(none))); }
template <int CTRL, int ROWS>
__device__ __forceinline__ double smp_move(double v, double none) {
  return __builtin_bit_cast(double, smp_move<CTRL, ROWS>(__builtin_bit_cast(smp_u64, v), __builtin_bit_cast(smp_u64, none)));
}
template <typename T, typename F>
__device__ __forceinline__ T smp_upto(T v, T none, F&& f) {
  v = f(v, smp_move<0x111, 0xf>(v, none));     // row_shr:1, 2, 4, 8
  v = f(v, smp_move<0x112, 0xf>(v, none));
  v = f(v, smp_move<0x114, 0xf>(v, none));
  v = f(v, smp_move<0x118, 0xf>(v, none));
  v = f(v, smp_move<0x142, 0xa>(v, none));     // row_bcast:15, row_bcast:31
  return f(v, smp_move<0x143, 0xc>(v, none));
}
__device__ __forceinline__ uint32_t smp_lane(uint32_t v, int lane) { return uint32_t(__builtin_amdgcn_readlane(int(v), lane)); }
__device__ __forceinline__ float smp_lane(float v, int lane) { return __uint_as_float(smp_lane(__float_as_uint(v), lane)); }
__device__ __forceinline__ smp_u64 smp_lane(smp_u64 v, int lane) { return smp_u64(smp_lane(uint32_t(v >> 32), lane)) << 32 | smp_lane(uint32_t(v), lane); }
template <typename T> __device__ __forceinline__ T smp_wave_upto(T v) { return smp_upto(v, T(0), [](T a, T b) { return a + b; }); }       // inclusive
template <typename T> __device__ __forceinline__ T smp_wave_sum(T v) { return smp_lane(smp_wave_upto(v), 63); }
__device__ __forceinline__ uint32_t smp_wave_max(uint32_t v) { return smp_lane(smp_upto(v, 0u, [](uint32_t a, uint32_t b) { return max(a, b); }), 63); }
__device__ __forceinline__ float smp_wave_max(float v) { return smp_lane(smp_upto(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); }), 63); }

// What is asked of a row.
struct SmpAsk {
  float T, p, least;
  int k;                             // 0: all
  bool greedy, filtered, cuts;
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
    cuts = k > 0 || p < 1.f;
    filtered = !greedy && (cuts || least > 0.f);
  }
};

// Largest logit of the row, by all lanes of a wave; *mine: that of chunk `lane`.
__device__ __forceinline__ float smp_row_top(const SampleChunk* of_row, int chunks, float* mine) {
  const int lane = threadIdx.x & 63;
  *mine = lane < chunks ? of_row[lane].top : -INFINITY;
  float top = *mine;
  for (int c = lane + 64; c < chunks; c += 64) top = fmaxf(top, of_row[c].top);
  return smp_wave_max(top);
}

template <bool BF16, int P>
__global__ __launch_bounds__(SMP_THREADS) void k_sample_chunks(SampleArgs a) {
  __shared__ double powers[256];
  __shared__ float tops[8];
  __shared__ uint32_t firsts[8], count[SMP_BINS][SMP_COPIES];
  __shared__ smp_u64 mass[SMP_BINS][SMP_COPIES];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, s = blockIdx.y, chunk = blockIdx.x;
  SampleChunk& out = a.chunk[static_cast<size_t>(s) * a.chunks + chunk];
  float v[P][4];
  smp_load<BF16, P>(a, s, chunk, v);
  if (tid < 256) powers[tid] = SMP_POWERS.v[tid];
  const SmpAsk ask(a, s);
  for (int i = tid; i < SMP_BINS * SMP_COPIES; i += SMP_THREADS) { (&count[0][0])[i] = 0; (&mass[0][0])[i] = 0; }
  float top = -INFINITY, most[P];              // of the chunk, of 256 neighbours
#pragma unroll
  for (int j = 0; j < P; ++j) {
    most[j] = smp_wave_max(fmaxf(fmaxf(v[j][0], v[j][1]), fmaxf(v[j][2], v[j][3])));
    top = fmaxf(top, most[j]);
  }
  if (lane == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) top = fmaxf(top, tops[w]);
  if (tid == 0) out.top = top;
  if (ask.greedy) {                            // the first index of the largest
    uint32_t first = ~0u;
#pragma unroll
    for (int j = P - 1; j >= 0; --j)
#pragma unroll
      for (int e = 3; e >= 0; --e)
        if (v[j][e] == top) first = uint32_t((chunk * P + j) * (SMP_THREADS * 4) + tid * 4 + e);
    first = ~smp_wave_max(~first);
    if (lane == 0) firsts[wave] = first;
    __syncthreads();
    if (tid == 0) {
#pragma unroll
      for (int w = 0; w < 8; ++w) first = min(first, firsts[w]);
      out.top_at = first;
    }
    return;
  }
  const double per = SmpScale::per_logit(ask.T);
  if (!ask.filtered) {                         // a chunk of nothing says so too
    const size_t block = static_cast<size_t>(s) * a.blocks + chunk * (P * 8) + wave;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      double sum = 0;                          // integers below 2^53: exact in any order
      if (most[j] > -INFINITY) {
        const SmpScale bs(per, most[j]);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += bs.mass_bits(bs.clean(v[j][e]), powers) - 4503599627370496.0;
        sum = smp_wave_upto(sum);
      }
      if (lane == 63) {
        a.block[block + j * 8] = static_cast<smp_u64>(sum);
        a.block_top[block + j * 8] = most[j];
      }
    }
    return;
  }
  if (top == -INFINITY || !ask.cuts) return;
  const SmpScale sc(per, top);
#pragma unroll
  for (int j = 0; j < P; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = sc.clean(v[j][e]);
      if (x > -INFINITY) {
        const int b = sc.bin(x);
        atomicAdd(&count[b][lane % SMP_COPIES], 1u);
        if (ask.p < 1.f && b < SMP_BINS - 1) atomicAdd(&mass[b][lane % SMP_COPIES], sc.bin_mass(x, powers));
      }
    }
  __syncthreads();
  if (tid < SMP_BINS) {
    uint32_t n = 0;
    smp_u64 m = 0;
#pragma unroll
    for (int c = 0; c < SMP_COPIES; ++c) { n += count[tid][c]; m += mass[tid][c]; }
    out.count[tid] = n;
    out.mass[tid] = m;
  }
}

template <bool BF16, int P>
__global__ __launch_bounds__(SMP_THREADS) void k_sample_cut(SampleArgs a) {
  constexpr int BLOCKS = P * 8, SEGMENTS = SMP_BINS / 64;
  __shared__ double powers[256];
  __shared__ smp_u64 mass[8][64];
  __shared__ uint32_t count[8][64], before[BLOCKS];
  __shared__ int bins_down[SMP_CHUNKS];
  __shared__ SampleRow cut;
  __shared__ uint32_t list_at;
  __shared__ int done;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, s = blockIdx.y, chunk = blockIdx.x;
  const SampleChunk* of_row = a.chunk + static_cast<size_t>(s) * a.chunks;
  float chunk_top;
  const float top = smp_row_top(of_row, a.chunks, &chunk_top);
  const SmpAsk ask(a, s);
  if (!ask.filtered || top == -INFINITY) return;
  float v[P][4];
  smp_load<BF16, P>(a, s, chunk, v);
  if (tid >= 256) powers[tid - 256] = SMP_POWERS.v[tid - 256];
  const double per = SmpScale::per_logit(ask.T);
  const SmpScale sc(per, top);
  if (sc.infinite) {
#pragma unroll
    for (int j = 0; j < P; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[j][e] = sc.clean(v[j][e]);
  }
  if (ask.cuts) {
    if (tid < a.chunks) {
      const float t = tid < 64 ? chunk_top : of_row[tid].top;
      bins_down[tid] = t > -INFINITY ? sc.bin_shift(SmpScale(per, t)) : SMP_BINS;
    }
    __syncthreads();
    // The row's bins, 64 at a time (16 octaves, mostly enough for top-k; top-p alone asks for the weight of all): wave w adds up those of every eighth chunk, wave 0 looks for the cuts.  What a
    // shift puts past the last bin weighs nothing and is not counted, and neither does the last bin's weight, which some chunks have and others not.
    SampleRow r{};
    r.k_bin = r.p_lo = SMP_BINS;
    r.p_hi = -1;
    smp_u64 n[SEGMENTS], m[SEGMENTS];          // of wave 0: sums up to bin 64 g + lane, weights in units of the row
#pragma unroll
    for (int g = 0; g < SEGMENTS; ++g) {
      smp_u64 mm = 0;
      uint32_t nn = 0;
#pragma unroll 4
      for (int c = wave; c < a.chunks; c += 8) {
        const int from = g * 64 + lane - bins_down[c];
        if (from >= 0) {
          nn += of_row[c].count[from];
          if (ask.p < 1.f) mm += of_row[c].mass[from];
        }
      }
      count[wave][lane] = nn;
      mass[wave][lane] = mm;
      __syncthreads();
      if (wave == 0) {
        n[g] = m[g] = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) { n[g] += count[w][lane]; m[g] += mass[w][lane]; }
        m[g] = g * 64 + lane < SMP_BINS - 1 ? m[g] >> sc.bin_unit_shift(g * 64 + lane) : 0;
        n[g] = smp_wave_upto(n[g]) + (g ? smp_lane(n[g > 0 ? g - 1 : 0], 63) : 0);
        m[g] = smp_wave_upto(m[g]) + (g ? smp_lane(m[g > 0 ? g - 1 : 0], 63) : 0);
        const smp_u64 so_far = smp_lane(n[g], 63);
        if (lane == 0) done = (ask.k > 0 && so_far >= static_cast<smp_u64>(ask.k)) || g + 1 == SEGMENTS ? g + 1 : 0;
      }
      __syncthreads();
      if (done) break;
    }
    if (wave == 0) {
      const int have = done;
      auto first = [&](auto&& reached) {         // first bin with reached(sums up to it), which holds for all after it; SMP_BINS - 1 if none
        int b = SMP_BINS - 1;
#pragma unroll
        for (int g = SEGMENTS - 1; g >= 0; --g)
          if (g < have) {
            const smp_u64 hit = __ballot(reached(n[g], m[g]));
            if (hit) b = g * 64 + __builtin_ctzll(hit);
          }
        return b;
      };
      auto before_bin = [&](const smp_u64 (&x)[SEGMENTS], int bin) {        // sum over the bins before it
        smp_u64 sum = 0;
#pragma unroll
        for (int g = 0; g < SEGMENTS; ++g)
          if (bin > 0 && (bin - 1) / 64 == g) sum = smp_lane(x[g], (bin - 1) & 63);
        return sum;
      };
      smp_u64 least = have == SEGMENTS ? smp_lane(m[SEGMENTS - 1], 63) : 0, most = least;       // weight that top-k leaves
      if (ask.k > 0) {
        r.k_bin = first([&](smp_u64 cn, smp_u64) { return cn >= static_cast<smp_u64>(ask.k); });
        if (r.k_bin == SMP_BINS - 1) {           // what is beyond weighs nothing
          r.k_bin = SMP_BINS;
        } else {
          r.k_above = before_bin(n, r.k_bin);
          least = before_bin(m, r.k_bin);
          most = before_bin(m, r.k_bin + 1);
        }
      }
      r.k_mass = least;
      if (ask.p < 1.f) {
        const double lo = double(ask.p) * double(least), hi = double(ask.p) * double(most);
        r.p_lo = first([&](smp_u64, smp_u64 cm) { return double(cm) >= lo && cm > 0; });
        r.p_hi = first([&](smp_u64, smp_u64 cm) { return double(cm) >= hi && cm > 0; });
        if (r.k_bin < SMP_BINS) { r.p_lo = min(r.p_lo, r.k_bin); r.p_hi = min(r.p_hi, r.k_bin); }
        r.p_mass = before_bin(m, r.p_lo);
      }
      // elements of the cuts' bins: in the row, and in the chunks ahead of this one
      const bool k_apart = r.k_bin < SMP_BINS && r.k_bin > r.p_hi;
      smp_u64 listed = r.p_hi >= 0 ? before_bin(n, r.p_hi + 1) - before_bin(n, r.p_lo) : 0;
      if (k_apart) listed += before_bin(n, r.k_bin + 1) - r.k_above;
      r.listed = int(listed);
      uint32_t ahead = 0;
      for (int c = lane; c < chunk; c += 64) {
        const int db = bins_down[c];
        for (int b = max(r.p_lo, db); b <= r.p_hi; ++b) ahead += of_row[c].count[b - db];
        if (k_apart && r.k_bin >= db) ahead += of_row[c].count[r.k_bin - db];
      }
      ahead = smp_wave_sum(ahead);
      if (lane == 0) {
        cut = r;
        list_at = ahead;
        if (chunk == 0) a.row[s] = r;
      }
    }
  } else if (tid == 0) {
    cut = SampleRow{SMP_BINS, SMP_BINS, -1, 0, 0, 0, 0};
    if (chunk == 0) a.row[s] = cut;
  }
  __syncthreads();
  // bins as ranges of 4 t: bin b is [floor4 - b, floor4 - b + 1), the last one all below it
  const int k_bin = cut.k_bin, p_lo = cut.p_lo, p_hi = cut.p_hi, sure = min(k_bin, p_lo);
  auto from = [&](int b) { return b >= SMP_BINS - 1 ? -INFINITY : sc.floor4 - b; };
  auto behind = [&](int b) { return b >= SMP_BINS ? -INFINITY : b <= 0 ? INFINITY : sc.floor4 - b + 1; };      // the first one has no end: where t is far from 0 a 1 more may be lost
  const double sure_from = sure >= SMP_BINS ? -INFINITY : behind(sure), p_from = from(p_hi), p_end = p_hi < 0 ? -INFINITY : behind(p_lo), k_from = from(k_bin), k_end = behind(k_bin);
  const double floor_t = ask.least > 0.f ? log2(double(ask.least)) : -INFINITY;
  smp_u64* block = a.block + static_cast<size_t>(s) * a.blocks + chunk * BLOCKS + wave;
  uint32_t mine[P];                              // bits of the elements to be listed
#pragma unroll
  for (int j = 0; j < P; ++j) {
    double sum = 0;
    mine[j] = 0;
    bool in[4], any = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const double t4 = double(v[j][e]) * sc.c * 4;
      const bool there = v[j][e] > -INFINITY;
      in[e] = there && t4 >= sure_from;
      any |= in[e];
      if (there && ((t4 >= k_from && t4 < k_end) || (t4 >= p_from && t4 < p_end))) mine[j] |= 1u << e;
    }
    if (__any(any)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += in[e] && sc.below(v[j][e]) >= floor_t ? sc.mass_bits(v[j][e], powers) - 4503599627370496.0 : 0.0;
      sum = smp_wave_upto(sum);
    }
    if (lane == 63) block[j * 8] = static_cast<smp_u64>(sum);
    const uint32_t n = uint32_t(__popcll(__ballot(mine[j] & 1)) + __popcll(__ballot(mine[j] & 2)) + __popcll(__ballot(mine[j] & 4)) + __popcll(__ballot(mine[j] & 8)));
    if (lane == 0) before[j * 8 + wave] = n;
  }
  if (cut.listed == 0 || cut.listed > a.list_size) return;
  __syncthreads();
  uint2* list = a.list + static_cast<size_t>(s) * a.list_size;
  const uint32_t ahead_of = smp_wave_upto(lane < BLOCKS ? before[lane] : 0u);
#pragma unroll
  for (int j = 0; j < P; ++j) {
    if (!__any(mine[j] != 0)) continue;
    const int b = __builtin_amdgcn_readfirstlane(j * 8 + wave);
    uint32_t at = list_at + (b ? smp_lane(ahead_of, b - 1) : 0u) + smp_wave_upto(uint32_t(__popc(mine[j]))) - __popc(mine[j]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if ((mine[j] >> e & 1) && at < uint32_t(a.list_size)) list[at++] = make_uint2(__float_as_uint(v[j][e]), uint32_t((chunk * P + j) * (SMP_THREADS * 4) + tid * 4 + e));
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

// Code that runs once is mostly the time of its instructions' way here: loops are not unrolled, and both cuts go through the same code.
template <bool BF16>
__global__ __launch_bounds__(SMP_THREADS) void k_sample_draw(SampleArgs a) {
  constexpr int KEYS = 1024;
  __shared__ double powers[256];
  __shared__ smp_u64 part[8], hist[KEYS], blocks[SMP_BLOCKS], found, found_here;
  __shared__ uint2 held[SMP_HELD];
  __shared__ uint32_t lows[8], highs[8];
  __shared__ int found_at;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, s = blockIdx.x, V = a.V;
  const SmpGroup group{part};
  const SampleChunk* of_row = a.chunk + static_cast<size_t>(s) * a.chunks;
  const int n_blocks = a.blocks;
  const smp_u64* row_blocks = a.block + static_cast<size_t>(s) * n_blocks;
  const float* block_tops = a.block_top + static_cast<size_t>(s) * n_blocks;
  const smp_u64 first_blocks = tid < n_blocks ? row_blocks[tid] : 0;        // asked for before it is known how they count
  float chunk_top;
  const float top = smp_row_top(of_row, a.chunks, &chunk_top);
  const SmpAsk ask(a, s);
  if (tid < 256) powers[tid] = SMP_POWERS.v[tid];
  if (top == -INFINITY) {
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

  // kept: logits above `cut`, and those equal to it before index `bound`
  float cut = -INFINITY;
  int bound = V;
  SampleRow r{SMP_BINS, SMP_BINS, -1, 0, 0, 0, 0};
  if (ask.filtered) r = a.row[s];
  const uint2* list = a.list + static_cast<size_t>(s) * a.list_size;
  const bool in_lds = r.listed <= SMP_HELD, in_list = r.listed <= a.list_size;
  if (in_lds && in_list)
    for (int i = tid; i < r.listed; i += SMP_THREADS) held[i] = list[i];
  __syncthreads();
  for (int b = tid; b < n_blocks; b += SMP_THREADS) {
    const smp_u64 x = b == tid ? first_blocks : row_blocks[b];
    int down = 0;
    if (!ask.filtered) {
      const float t = block_tops[b];
      down = t > -INFINITY ? sc.unit_shift(SmpScale(per, t)) : 64;
    }
    blocks[b] = down < 64 ? x >> down : 0;
  }
  if (r.listed > 0) {
    const int n = in_list ? r.listed : V;
    auto each = [&](auto&& f) {                  // f(logit, index) of every element of the bins in question, and others of the row where there is no list
#pragma unroll 1
      for (int i = tid; i < n; i += SMP_THREADS) {
        const uint2 y = !in_list ? make_uint2(__float_as_uint(sc.clean(smp_one<BF16>(a, s, i))), uint32_t(i)) : in_lds ? held[i] : list[i];
        const float x = __uint_as_float(y.x);
        if (x > -INFINITY) f(x, int(min(y.y, uint32_t(V - 1))));
      }
    };
    smp_u64 whole = r.k_mass;                    // weight that top-k leaves
    int b_lo = 0, b_hi = 0, k_bound = bound;
    float k_cut = cut;
    smp_u64 target = 0;
    bool indexes = false;
#pragma unroll 1
    for (int stage = 0; stage < 4; ++stage) {    // top-k by counts, the elements equal to its cut by index, top-p by weights, those equal to its cut
      const bool by_mass = stage == 2, by_index = stage & 1;
      if (by_index ? !indexes : by_mass ? !(ask.p < 1.f) : r.k_bin == SMP_BINS) continue;
      if (!by_index) {
        if (by_mass && r.k_bin < SMP_BINS) {
          smp_u64 m = 0;
          each([&](float x, int i) {
            if (sc.bin(x) == r.k_bin && (x > cut || (x == cut && i < bound))) m += sc.mass(x, powers);
          });
          whole = r.k_mass + group.sum(m);
          __syncthreads();
        }
        b_lo = by_mass ? r.p_lo : r.k_bin;
        b_hi = by_mass ? r.p_hi : r.k_bin;
        k_cut = cut;
        k_bound = bound;
        const double goal = double(ask.p) * double(whole) - double(r.p_mass);
        target = !by_mass ? static_cast<smp_u64>(ask.k) - r.k_above : goal > 1. ? static_cast<smp_u64>(ceil(goal)) : 1;       // the first one is kept always
      }
      indexes = false;
      auto in = [&](float x, int i) {
        const int b = sc.bin(x);
        return b >= b_lo && b <= b_hi && (x > k_cut || (x == k_cut && i < k_bound)) && (!by_index || x == cut);
      };
      auto key = [&](float x, int i) { return by_index ? ~uint32_t(i) : smp_key<BF16>(x); };
      // the largest key with the sum over it and those above it >= target
      uint32_t lo = ~0u, hi = 0;
      each([&](float x, int i) {
        if (in(x, i)) {
          const uint32_t k = key(x, i);
          lo = min(lo, k);
          hi = max(hi, k);
        }
      });
      lo = ~smp_wave_max(~lo);
      hi = smp_wave_max(hi);
      if (lane == 0) { lows[wave] = lo; highs[wave] = hi; }
      __syncthreads();
#pragma unroll
      for (int w = 0; w < 8; ++w) { lo = min(lo, lows[w]); hi = max(hi, highs[w]); }
      if (hi < lo) {
        __syncthreads();
        continue;
      }
      const uint32_t lowest = lo;
      smp_u64 over = 0, here = 0;                // sums above the bin in question and in it
      bool reached = true;
#pragma unroll 1
      while (true) {
        const int shift = max(0, 32 - __builtin_clz((hi - lo) | 1) - 10);
        hist[2 * tid] = hist[2 * tid + 1] = 0;
        if (tid == 0) found_at = KEYS;
        __syncthreads();
        each([&](float x, int i) {
          const uint32_t k = key(x, i);
          if (k >= lo && k <= hi && in(x, i)) {
            const smp_u64 w = by_mass ? sc.mass(x, powers) : 1;
            if (w) atomicAdd(&hist[(hi - k) >> shift], w);
          }
        });
        __syncthreads();
        const smp_u64 one = hist[2 * tid], two = hist[2 * tid + 1], upto = over + group.upto(one + two), ahead = upto - one - two;
        if (upto >= target && ahead < target) {  // one thread at most
          const bool second = ahead + one < target;
          found_at = 2 * tid + second;
          found = ahead + (second ? one : 0);
          found_here = second ? two : one;
        }
        __syncthreads();
        const int bin = found_at;
        if (bin == KEYS) { reached = false; break; }
        over = found;
        here = found_here;
        hi -= uint32_t(bin) << shift;
        lo = shift ? max(lo, hi - ((1u << shift) - 1)) : hi;
        __syncthreads();
        if (shift == 0) break;
      }
      __syncthreads();
      if (by_index) {
        bound = reached ? int(~hi) + 1 : bound;  // behind the last one that is kept
        continue;
      }
      cut = smp_value<BF16>(reached ? hi : lowest);       // not reached, for want of the last units: all of these bins
      bound = cut == k_cut ? k_bound : V;
      if (reached) {                             // of the elements equal to the cut so many
        const smp_u64 w = by_mass ? sc.mass(cut, powers) : 1;
        target = (target - over + w - 1) / w;
        indexes = target * w < here;
      }
    }
    // what is kept of those bins joins the sums of its neighbourhoods
    const int sure = min(r.k_bin, r.p_lo);
    each([&](float x, int i) {
      const int b = sc.bin(x);
      if (b < sure || (b != r.k_bin && (b < r.p_lo || b > r.p_hi))) return;
      if ((x > cut || (x == cut && i < bound)) && sc.below(x) >= floor_t) atomicAdd(&blocks[i / SMP_NEIGHBOURS], sc.mass(x, powers));
    });
  }
  __syncthreads();

  // the neighbourhood: a thread has some that follow one another
  const int each_t = (n_blocks + SMP_THREADS - 1) / SMP_THREADS, b0 = min(n_blocks, tid * each_t), b1 = min(n_blocks, b0 + each_t);
  smp_u64 mine = 0;
  for (int b = b0; b < b1; ++b) mine += blocks[b];
  const smp_u64 upto = group.upto(mine);
  if (tid == SMP_THREADS - 1) found = upto;
  __syncthreads();
  const smp_u64 W = found;
  float u = a.u[s];
  u = u > 0.f ? fminf(u, 1.f) : 0.f;
  // the first running weight above u W; in integers: of at least floor(u W) + 1, and W where u is 1
  smp_u64 goal = static_cast<smp_u64>(floor(double(u) * double(W))) + 1;
  goal = goal > W ? W : goal;
  if (tid == 0) found_at = 0;
  __syncthreads();
  if (upto >= goal && upto - mine < goal) {
    smp_u64 run = upto - mine;
    int b = b0;
    while (b + 1 < b1 && run + blocks[b] < goal) run += blocks[b++];
    found_at = b;
    found = goal - run;
  }
  __syncthreads();
  if (wave != 0) return;
  const int block = found_at;
  goal = found;
  // The same weights in the same units again, shifted as their sum was: the running weight of the last one is the neighbourhood's.
  const SmpScale bs(per, ask.filtered ? top : block_tops[block]);
  const int down = sc.unit_shift(bs);
  float x[4];
  smp_u64 m[4], own = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int i = block * SMP_NEIGHBOURS + lane * 4 + e;
    x[e] = i < V ? smp_one<BF16>(a, s, i) : -INFINITY;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int i = block * SMP_NEIGHBOURS + lane * 4 + e;
    x[e] = sc.clean(x[e]);
    const bool in = (x[e] > cut || (x[e] == cut && i < bound)) && sc.below(x[e]) >= floor_t;
    m[e] = in && x[e] > -INFINITY ? bs.mass(x[e], powers) : 0;
    own += m[e];
  }
  const smp_u64 run_upto = smp_wave_upto(own);
  if ((run_upto >> down) >= goal && ((run_upto - own) >> down) < goal) {
    smp_u64 run = run_upto - own;
    int e = 0;
    while (e < 3 && ((run + m[e]) >> down) < goal) run += m[e++];
    const float v = e == 0 ? x[0] : e == 1 ? x[1] : e == 2 ? x[2] : x[3];
    a.tokens[s] = block * SMP_NEIGHBOURS + lane * 4 + e;
    if (a.logprobs) {
      // Of a token with half of the weight or more, by what is not its: integers, 0 where it is the only one.  Of others, by their weight before it was rounded: that may be far below a unit.
      const smp_u64 one = e == 0 ? m[0] : e == 1 ? m[1] : e == 2 ? m[2] : m[3];
      const double rest = fmax(ldexp(double(W), down) - double(one), 0.0);
      a.logprobs[s] = float(rest <= double(one) ? 0.0 - log1p(rest / double(one)) : (sc.units(v) - log2(double(W))) * 0.69314718055994530942);
    }
  }
}

namespace {
struct SampleSpace { int places, chunks, list_size; size_t row, block, block_top, list, total; };
SampleSpace space(int S, int V) {
  SampleSpace p;
  p.places = static_cast<long long>(S) * V < (1 << 21) && V <= SMP_CHUNKS * SMP_THREADS * 4 ? 1 : 4;
  p.chunks = (V + p.places * SMP_THREADS * 4 - 1) / (p.places * SMP_THREADS * 4);
  p.row = align256(size_t(S) * p.chunks * sizeof(SampleChunk));
  p.block = p.row + align256(size_t(S) * sizeof(SampleRow));
  p.block_top = p.block + align256(size_t(S) * p.chunks * p.places * 8 * 8);
  p.list = p.block_top + align256(size_t(S) * p.chunks * p.places * 8 * 4);
  p.list_size = V < SMP_LIST ? V : SMP_LIST;
  p.total = p.list + align256(size_t(S) * p.list_size * 8);
  return p;
}
}  // namespace

size_t sample_ws_bytes(int S, int V) { return space(S, V).total; }

int32_t launch_sample(const void* logits, bool bf16, long long stride, int S, int V, const moqe_sampling& how, const float* u, int32_t* tokens, float* logprobs,
                      void* ws, hipStream_t st) {
  const SampleSpace p = space(S, V);
  uint8_t* b = static_cast<uint8_t*>(ws);
  SampleArgs a{logits, stride, how.temperature, how.top_k, how.top_p, how.min_p, u, tokens, logprobs, S, V, p.chunks, p.chunks * p.places * 8, p.list_size,
               reinterpret_cast<SampleChunk*>(b), reinterpret_cast<SampleRow*>(b + p.row), reinterpret_cast<smp_u64*>(b + p.block), reinterpret_cast<float*>(b + p.block_top),
               reinterpret_cast<uint2*>(b + p.list)};
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
