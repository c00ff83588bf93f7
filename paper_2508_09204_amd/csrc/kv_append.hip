// Rotary positions of a fused projection's query and key heads, keys and values into the paged cache of e4m3 codes.
#include "kv_device.h"

namespace moqe {

struct AppendArgs {
  const void* qkv; uint16_t* q;
  long long qkv_stride, q_stride;
  KvBatch b; KvCache c;
  const double* inv_freq; const float *q_gain, *k_gain;
  float eps, mscale;
  int heads, rot, inter;
  int seq_blocks;               // cache part: blocks that a sequence of T rows can touch, ...
  int key_groups, group_heads;  // ... key heads in groups that a work-group goes through
  int row_tiles, rows_log2;     // query part: tiles of 2^rows_log2 rows of a sequence, ...
  int splits, split_heads;      // ... its heads in parts
};

// Rows are taken in pieces of 16 bytes: PIECE values.  A slot is two pieces of a head vector that hold whole pairs of the rotation; a head's DH / (2 PIECE) slots
// lie in neighbouring lanes, so that a load of first (second) pieces covers a stretch of memory without holes.
template <bool BF16> constexpr int PIECE = BF16 ? 8 : 4;
template <int DH, bool BF16> constexpr int SLOTS = DH / (2 * PIECE<BF16>);

template <int DH, bool BF16>
__device__ __forceinline__ void slot_dims(const AppendArgs& a, int slot, int* da, int* db) {
  constexpr int P = PIECE<BF16>;
  if (a.inter || a.rot == DH) {                 // pairs within pieces, or of pieces half a head apart
    *da = slot * P;
    *db = slot * P + DH / 2;
  } else if (slot * 2 * P < a.rot) {            // pairs of pieces rot / 2 apart
    *da = slot * P;
    *db = slot * P + a.rot / 2;
  } else {
    *da = slot * 2 * P;
    *db = slot * 2 * P + P;
  }
}

// cos and sin of angle number j at position p, rounded once: all is done in 64 bits, where 32 would lose 2^-24 of p * inv_freq, and an error in the last places of cos and sin
// moves keys over the borders between codes.  The angle is taken to its fraction of a turn, that to the nearest quarter; on what is left, up to pi / 4, the power series
// to x^11 and x^10 leave 2^-33.
__device__ __forceinline__ void angle(const AppendArgs& a, int j, int p, float* cs, float* sn) {
  double turns = double(p) * (a.inv_freq[j] * 0.15915494309189535);
  turns -= rint(turns);
  const double quarters = rint(4.0 * turns), x = fma(-0.25, quarters, turns) * 6.283185307179586, z = x * x;
  const double s = x * fma(z, fma(z, fma(z, fma(z, fma(z, -1.0 / 39916800, 1.0 / 362880), -1.0 / 5040), 1.0 / 120), -1.0 / 6), 1.0);
  const double c = fma(z, fma(z, fma(z, fma(z, fma(z, -1.0 / 3628800, 1.0 / 40320), -1.0 / 720), 1.0 / 24), -0.5), 1.0);
  const int n = static_cast<int>(quarters) & 3;
  const float fs = float(s * double(a.mscale)), fc = float(c * double(a.mscale));
  const float u = n & 1 ? fs : fc, v = n & 1 ? fc : fs;
  *cs = n == 1 || n == 2 ? -u : u;
  *sn = n >= 2 ? -v : v;
}
// Which of a slot's pieces the rotation takes: with neighbouring pairs each by itself, in the half layout both or none.  rot is a multiple of 16, so a piece is in or out as a whole.
struct SlotTurns { bool first, second; };
__device__ __forceinline__ SlotTurns slot_turns(const AppendArgs& a, int da, int db) {
  if (a.inter) return SlotTurns{da < a.rot, db < a.rot};
  const bool both = da < a.rot / 2;
  return SlotTurns{both, both};
}

template <int P>
__device__ __forceinline__ void slot_angles(const AppendArgs& a, int da, int db, int p, float* cs, float* sn) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const bool second = a.inter && i >= P / 2;
    const int dim = a.inter ? (second ? db : da) + 2 * (i % (P / 2)) : da + i;
    cs[i] = 1.f;
    sn[i] = 0.f;
    if (dim < (a.inter ? a.rot : a.rot / 2)) angle(a, a.inter ? dim / 2 : dim, p, &cs[i], &sn[i]);
    __builtin_amdgcn_sched_barrier(0);           // one after the other: side by side they would take the registers of two more waves
  }
}

// e cos - f sin.  EXACT: with what the rounding of f sin leaves, so that the result is rounded once.
template <bool EXACT>
__device__ __forceinline__ float turned(float e, float f, float cs, float sn) {
  const float w = f * sn, r = fmaf(e, cs, -w);
  if (!EXACT) return r;
  const float x = r - fmaf(f, sn, -w);
  return x == x ? x : r;                         // an infinite f leaves NaN
}
// Pieces that the rotation leaves out have cos 1 and sin 0, and a partner of 0: an infinity or NaN times that sin would be NaN.
template <int P, bool EXACT>
__device__ __forceinline__ void turn(bool inter, const SlotTurns& on, const float* cs, const float* sn, float* x) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const bool turns = i < P / 2 ? on.first : on.second;
    const int s = i, t = P + i;                                       // half layout
    const int u = i / (P / 2) * P + 2 * (i % (P / 2));                // neighbours
    if (inter) {
      const float e = x[u], f = x[u + 1];
      x[u] = turned<EXACT>(e, turns ? f : 0.f, cs[i], sn[i]);
      x[u + 1] = turned<EXACT>(f, turns ? e : 0.f, cs[i], -sn[i]);
    } else {
      const float e = x[s], f = x[t];
      x[s] = turned<EXACT>(e, turns ? f : 0.f, cs[i], sn[i]);
      x[t] = turned<EXACT>(f, turns ? e : 0.f, cs[i], -sn[i]);
    }
  }
}

template <bool BF16>
__device__ __forceinline__ uint4 load_piece(const void* base, long long at) {
  return *reinterpret_cast<const uint4*>(static_cast<const char*>(base) + at * (BF16 ? 2 : 4));
}
template <bool BF16>
__device__ __forceinline__ void piece_values(const uint4& p, float* x) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      x[i] = __uint_as_float(w[i]);
    }
  }
}

// RMS norm of a head vector whose slots lie in neighbouring lanes.  EXACT: what follows the sum of squares is rounded twice only.
template <int DH, bool BF16, bool EXACT>
__device__ __forceinline__ void head_norm(const float* gain, float eps, int da, int db, float* x) {
  constexpr int P = PIECE<BF16>;
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < 2 * P; ++i) q += x[i] * x[i];
#pragma unroll
  for (int d = 1; d < SLOTS<DH, BF16>; d *= 2) q += __shfl_xor(q, d);
  float hi, lo = 0.f;
  if constexpr (EXACT) {
    const double inv = 1.0 / sqrt(double(q) / DH + double(eps));
    hi = float(inv);
    lo = float(inv - double(hi));
  } else {
    hi = 1.f / sqrtf(q / float(DH) + eps);
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const float ga = gain[da + i], gb = gain[db + i];
    x[i] *= EXACT ? fmaf(hi, ga, lo * ga) : hi * ga;
    x[P + i] *= EXACT ? fmaf(hi, gb, lo * gb) : hi * gb;
  }
}

// Codes of x / scale for a power of two, to nearest even; NaN stays, past 464 gets NaN.
__device__ __forceinline__ uint32_t codes4(const float* x, float scale) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  s16x2 w = {0, 0};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[0], x[1], scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[2], x[3], scale, true);
  return __builtin_bit_cast(uint32_t, w);
}
__device__ __forceinline__ uint32_t rescaled4(uint32_t w, float by) {
  const float x[4] = {__builtin_amdgcn_cvt_f32_fp8(w, 0) * by, __builtin_amdgcn_cvt_f32_fp8(w, 1) * by, __builtin_amdgcn_cvt_f32_fp8(w, 2) * by,
                      __builtin_amdgcn_cvt_f32_fp8(w, 3) * by};
  return codes4(x, 1.f);
}

// The codes of the tokens before `lo` of a block and head (first token `first`) move to a scale that is 1 / by times as large.
template <int DH>
__device__ __forceinline__ void rescale_block(uint8_t* codes, bool values, int bt, int first, int lo, float by) {
  for (int u = threadIdx.x; u < bt * DH / 16; u += blockDim.x) {
    // values: dword j of a unit is tokens t0 + 16 (j & 1) + 0 .. 3; keys: all of a unit is one token
    const int t0 = values ? first + u / (2 * DH) * 32 + u % 64 / 16 * 4 : first + u / DH * 16 + u % 16;
    if (t0 >= lo) continue;
    uint4* p = reinterpret_cast<uint4*>(codes) + u;
    uint4 w = *p;
    uint32_t* d = &w.x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int left = values ? lo - (t0 + 16 * (j & 1)) : 4;
      const uint32_t keep = left >= 4 ? 0u : left <= 0 ? ~0u : ~0u << (8 * left);
      d[j] = (rescaled4(d[j], by) & ~keep) | (d[j] & keep);
    }
    *p = w;
  }
}

// What the threads of a work-group find out about one block and head: the new scale, and what earlier codes have to be multiplied with (1: nothing).  top: the largest
// finite |x| of the thread.
struct BlockScale { float scale, by; };
__device__ __forceinline__ BlockScale block_scale(float top, bool held, float old, float* at, float* wave_max) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = top;
  __syncthreads();                               // also: everybody has read the old scale
  for (int w = 0; w < int(blockDim.x) / 64; ++w) top = fmaxf(top, wave_max[w]);
  const float need = __uint_as_float(uint32_t(kv_scale_exponent(__float_as_uint(top)) + 127) << 23);
  BlockScale s;
  s.scale = held && !(old < need) ? old : need;
  s.by = held && s.scale > old ? old * (1.f / s.scale) : 1.f;
  if (threadIdx.x == 0) *at = s.scale;
  return s;
}
// The largest finite |x| (NaN is passed over), and whether any is infinite: the conversion would make NaN of those.
template <int N>
__device__ __forceinline__ void largest(const float (&x)[N], float* top, bool* infinite) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, fabsf(x[i]));
  if (m == INFINITY) {
    *infinite = true;
    m = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (fabsf(x[i]) < INFINITY) m = fmaxf(m, fabsf(x[i]));
  }
  *top = fmaxf(*top, m);
}
// Infinities as what becomes the largest code by the scale returned: that given, or half of it, of values halved too, where 448 of it would be an infinity again.  All of a thread's values of a block
// have the same one.
template <int N>
__device__ __forceinline__ float no_infinities(float (&x)[N], bool infinite, float scale) {
  if (!infinite) return scale;
  const float by = 448.f * scale < INFINITY ? 1.f : 0.5f;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = fabsf(x[i]) == INFINITY ? copysignf(448.f * (scale * by), x[i]) : x[i] * by;
  return scale * by;
}

// A block of a sequence that a call writes to: its new tokens lo .. hi, its first token, its place in the cache.
struct BlockTokens {
  int lo, hi, first, id;
  long long row;                // of token lo
  bool held;                    // it held earlier tokens
};
__device__ __forceinline__ bool block_tokens(const AppendArgs& a, int s, int n, BlockTokens* b) {
  const KvSeq q = kv_seq(a.b, s, a.c.bt_log2);
  const int p0 = max(q.first(), 0), end = min(q.len, q.first() + min(q.n, a.b.T));
  const int blk = (p0 >> a.c.bt_log2) + n;
  b->first = blk << a.c.bt_log2;
  b->lo = max(p0, b->first);
  b->hi = min(end, b->first + (1 << a.c.bt_log2));
  if (b->lo >= b->hi) return false;
  b->id = a.b.table[static_cast<long long>(s) * a.b.width + blk];
  b->row = q.row0 + (b->lo - q.first());
  b->held = b->lo > b->first;
  return b->id >= 0 && b->id < a.c.n_blocks;
}

// Keys of one block for some heads in turn.  Their norm and rotation are kept to few roundings in fp32: each one moves some keys over the border between two codes.  A thread has 32 values in slots, the same tokens and dims for every head, so that it works out its angles once for all of them.
template <int DH, bool BF16>
__device__ __forceinline__ void append_keys(const AppendArgs& a, const BlockTokens& b, int head0, int head1, float (*wave_max)[16]) {
  constexpr int P = PIECE<BF16>, SL = SLOTS<DH, BF16>, NS = 16 / P;
  const int slots = (b.hi - b.lo) * SL, tid = threadIdx.x, th = blockDim.x;
  int da, db;
  slot_dims<DH, BF16>(a, tid % SL, &da, &db);
  const SlotTurns on = slot_turns(a, da, db);
  uint4 pa[NS], pb[NS];
  auto load = [&](int head) {
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const int u = n * th + tid;
      if (u < slots) {
        const long long at = (b.row + u / SL) * a.qkv_stride + static_cast<long long>(a.heads + head) * DH;
        pa[n] = load_piece<BF16>(a.qkv, at + da);
        pb[n] = load_piece<BF16>(a.qkv, at + db);
      }
    }
  };
  load(head0);
  float cs[NS][P], sn[NS][P];
  if (a.rot > 0) {
#pragma unroll
    for (int n = 0; n < NS; ++n)
      if (n * th + tid < slots) slot_angles<P>(a, da, db, b.lo + (n * th + tid) / SL, cs[n], sn[n]);
  }
  for (int head = head0; head < head1; ++head) {
    const long long bh = static_cast<long long>(b.id) * a.c.heads + head;
    uint8_t* codes = a.c.k + bh * (static_cast<long long>(DH) << a.c.bt_log2);
    const float old = b.held ? a.c.k_scale[bh] : 0.f;
    float x[NS][2 * P];
    float top = 0.f;
    bool infinite = false;
    // The gains are read again for every head: held through the loop, which they would be if the address were known to stay, they are the registers that spill (16 x 256 rows in bf16
    // with heads of 256, blocks of 128: 296 us and 1044 bytes of scratch a lane, so 58 and none).
    const float* gain = a.k_gain;
    asm("" : "+s"(gain));
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      if (n * th + tid < slots) {
        piece_values<BF16>(pa[n], x[n]);
        piece_values<BF16>(pb[n], x[n] + P);
        if (gain) head_norm<DH, BF16, true>(gain, a.eps, da, db, x[n]);        // a head vector's slots are all in or all out
        if (a.rot > 0) turn<P, true>(a.inter, on, cs[n], sn[n], x[n]);
        largest(x[n], &top, &infinite);
      }
    }
    if (head + 1 < head1) load(head + 1);
    const BlockScale s = block_scale(top, b.held, old, a.c.k_scale + bh, wave_max[(head - head0) & 1]);
    if (s.by != 1.f) {
      rescale_block<DH>(codes, false, 1 << a.c.bt_log2, b.first, b.lo, s.by);
      __syncthreads();                           // before parts of the same units are written
    }
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const int u = n * th + tid;
      if (u >= slots) continue;
      const float scale = no_infinities(x[n], infinite, s.scale);
      const uint32_t t = uint32_t(b.lo - b.first + u / SL);
      uint8_t* ka = codes + kv_key_at(t, uint32_t(da), DH);
      uint8_t* kb = codes + kv_key_at(t, uint32_t(db), DH);
      if constexpr (BF16) {
        *reinterpret_cast<uint2*>(ka) = make_uint2(codes4(x[n], scale), codes4(x[n] + 4, scale));
        *reinterpret_cast<uint2*>(kb) = make_uint2(codes4(x[n] + 8, scale), codes4(x[n] + 12, scale));
      } else {
        *reinterpret_cast<uint32_t*>(ka) = codes4(x[n], scale);
        *reinterpret_cast<uint32_t*>(kb) = codes4(x[n] + 4, scale);
      }
    }
  }
}

// Values of one block and head.  Their codes lie four tokens to a dword.  Where all 32 tokens of a group are new, a thread takes a piece of four rows and writes whole dwords,
// through LDS; the tokens of other groups go byte by byte.
template <int DH, bool BF16>
__device__ __forceinline__ void append_values(const AppendArgs& a, const BlockTokens& b, int head, uint32_t* lds, float* wave_max) {
  constexpr int P = PIECE<BF16>, PCS = DH / P, NQ = BF16 ? 1 : 2;
  const int tid = threadIdx.x, th = blockDim.x;
  const long long bh = static_cast<long long>(b.id) * a.c.heads + head;
  uint8_t* codes = a.c.v + bh * (static_cast<long long>(DH) << a.c.bt_log2);
  const long long col = static_cast<long long>(a.heads + a.c.heads + head) * DH;
  // groups g_lo .. g_hi are new altogether, the other new tokens are `before` from lo on and those from `behind` on
  const int g_lo = (b.lo - b.first + 31) / 32, g_hi = (b.hi - b.first) / 32;
  const bool whole = g_hi > g_lo;
  const int quads = whole ? (g_hi - g_lo) * 8 * PCS : 0;
  const int before = whole ? b.first + 32 * g_lo - b.lo : b.hi - b.lo, behind = whole ? b.first + 32 * g_hi : b.hi;
  const int rest = (before + b.hi - behind) * PCS;
  auto rest_token = [&](int u) { const int v = u / PCS; return v < before ? b.lo + v : behind + v - before; };
  auto rest_piece = [&](int u) { return load_piece<BF16>(a.qkv, (b.row + rest_token(u) - b.lo) * a.qkv_stride + col + u % PCS * P); };
  uint4 vq[NQ][4], vr;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int u = n * th + tid;
    if (u < quads) {
      const long long at = (b.row + b.first + 32 * g_lo + u / PCS * 4 - b.lo) * a.qkv_stride + col + u % PCS * P;
#pragma unroll
      for (int t = 0; t < 4; ++t) vq[n][t] = load_piece<BF16>(a.qkv, at + t * a.qkv_stride);
    }
  }
  if (tid < rest) vr = rest_piece(tid);
  const float old = b.held ? a.c.v_scale[bh] : 0.f;
  float top = 0.f;
  bool infinite = false;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    if (n * th + tid < quads) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        float x[P];
        piece_values<BF16>(vq[n][t], x);
        largest(x, &top, &infinite);
      }
    }
  }
  for (int u = tid; u < rest; u += th) {
    float x[P];
    piece_values<BF16>(u == tid ? vr : rest_piece(u), x);
    largest(x, &top, &infinite);
  }
  const BlockScale s = block_scale(top, b.held, old, a.c.v_scale + bh, wave_max);
  if (s.by != 1.f) {
    rescale_block<DH>(codes, true, 1 << a.c.bt_log2, b.first, b.lo, s.by);
    __syncthreads();                             // before single bytes of the same units are written
  }
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int u = n * th + tid;
    if (u < quads) {
      uint32_t* to = lds + kv_value_at(uint32_t(32 * g_lo + u / PCS * 4), uint32_t(u % PCS * P), DH) / 4;
      float x[4][P], scale;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        piece_values<BF16>(vq[n][t], x[t]);
        scale = no_infinities(x[t], infinite, s.scale);
      }
#pragma unroll
      for (int i = 0; i < P; ++i) {              // neighbouring dims of 16 lie 16 bytes apart
        const float y[4] = {x[0][i], x[1][i], x[2][i], x[3][i]};
        to[4 * i] = codes4(y, scale);
      }
    }
  }
  for (int u = tid; u < rest; u += th) {
    float x[P];
    piece_values<BF16>(u == tid ? vr : rest_piece(u), x);
    const float scale = no_infinities(x, infinite, s.scale);
    uint8_t* to = codes + kv_value_at(uint32_t(rest_token(u) - b.first), uint32_t(u % PCS * P), DH);
#pragma unroll
    for (int i = 0; i < P; i += 4) {
      const uint32_t w = codes4(x + i, scale);
#pragma unroll
      for (int t = 0; t < 4; ++t) to[16 * (i + t)] = uint8_t(w >> (8 * t));
    }
  }
  if (whole) {
    __syncthreads();
    for (int u = g_lo * 2 * DH + tid; u < g_hi * 2 * DH; u += th) reinterpret_cast<uint4*>(codes)[u] = reinterpret_cast<const uint4*>(lds)[u];
  }
}

// Work-groups of the keys (one for each block a sequence can touch and group of heads), of the values (one for each block and head), then of the queries (a row tile
// and some heads each).  At most TH threads: 1024 for blocks of 128 tokens of 256 dims, whose work-groups have to do with 128 registers.
// Bound by memory: 16 prompts of 512 tokens with 32 heads of 128 (336 MB) 75 us,
// rows of mixed lengths in fp32 with 28 (475 MB) 104 us, where a copy of as many bytes takes 68 and 96.
template <int DH, bool BF16, int TH>
__global__ __launch_bounds__(TH, TH > 512 ? 1 : BF16 ? 4 : 3) void k_kv_append(AppendArgs a) {
  extern __shared__ __align__(16) uint32_t lds[];
  __shared__ float wave_max[2][16];
  constexpr int P = PIECE<BF16>, SL = SLOTS<DH, BF16>;
  const int tid = threadIdx.x;
  int w = blockIdx.x;
  const int key_wgs = a.b.S * a.seq_blocks * a.key_groups, cache_wgs = key_wgs + a.b.S * a.seq_blocks * a.c.heads;
  if (w < cache_wgs) {
    const bool keys = w < key_wgs;
    w -= keys ? 0 : key_wgs;
    const int per = keys ? a.key_groups : a.c.heads, part = w % per, n = w / per;
    BlockTokens b;
    if (!block_tokens(a, n / a.seq_blocks, n % a.seq_blocks, &b)) return;
    if (keys) append_keys<DH, BF16>(a, b, part * a.group_heads, min(a.c.heads, (part + 1) * a.group_heads), wave_max);
    else append_values<DH, BF16>(a, b, part, lds, wave_max[0]);
    return;
  }
  w -= cache_wgs;
  const int split = w % a.splits, s = w / a.splits / a.row_tiles;
  const int lane_row = (tid / SL) & ((1 << a.rows_log2) - 1), group = tid / SL >> a.rows_log2, groups = blockDim.x / SL >> a.rows_log2;
  const KvSeq q = kv_seq(a.b, s, a.c.bt_log2);
  const int i = (w / a.splits % a.row_tiles << a.rows_log2) + lane_row;
  if (i >= min(q.n, a.b.T)) return;
  int da, db;
  slot_dims<DH, BF16>(a, tid % SL, &da, &db);
  const SlotTurns on = slot_turns(a, da, db);
  const long long row = static_cast<long long>(q.row0 + i) * a.qkv_stride, to = (q.row0 + i) * a.q_stride;
  const int h_end = min(a.heads, (split + 1) * a.split_heads);
  constexpr int B = 4;                           // heads in flight
  float cs[P], sn[P];
  bool known = false;
  for (int h0 = split * a.split_heads + group; h0 < h_end; h0 += B * groups) {
    uint4 pa[B], pb[B];
#pragma unroll
    for (int n = 0; n < B; ++n) {
      const int h = h0 + n * groups;
      if (h < h_end) {
        pa[n] = load_piece<BF16>(a.qkv, row + h * DH + da);
        pb[n] = load_piece<BF16>(a.qkv, row + h * DH + db);
      }
    }
    if (!known && a.rot > 0) slot_angles<P>(a, da, db, q.first() + i, cs, sn);
    known = true;
#pragma unroll
    for (int n = 0; n < B; ++n) {
      const int h = h0 + n * groups;
      if (h >= h_end) continue;
      float x[2 * P];
      piece_values<BF16>(pa[n], x);
      piece_values<BF16>(pb[n], x + P);
      if (a.q_gain) head_norm<DH, BF16, false>(a.q_gain, a.eps, da, db, x);
      if (a.rot > 0) turn<P, false>(a.inter, on, cs, sn, x);
      uint16_t* oa = a.q + to + h * DH + da;
      uint16_t* ob = a.q + to + h * DH + db;
      if constexpr (BF16) {
        *reinterpret_cast<uint4*>(oa) = make_uint4(kv_pair(x[0], x[1]), kv_pair(x[2], x[3]), kv_pair(x[4], x[5]), kv_pair(x[6], x[7]));
        *reinterpret_cast<uint4*>(ob) = make_uint4(kv_pair(x[8], x[9]), kv_pair(x[10], x[11]), kv_pair(x[12], x[13]), kv_pair(x[14], x[15]));
      } else {
        *reinterpret_cast<uint2*>(oa) = make_uint2(kv_pair(x[0], x[1]), kv_pair(x[2], x[3]));
        *reinterpret_cast<uint2*>(ob) = make_uint2(kv_pair(x[4], x[5]), kv_pair(x[6], x[7]));
      }
    }
  }
}


int32_t launch_kv_append(const void* qkv, bool bf16, long long qkv_stride, int heads, const moqe_rope& r, const moqe_kv_batch& b,
                         const moqe_kv_cache& c, void* q_out, long long q_stride, hipStream_t st) {
  AppendArgs a{};
  a.qkv = qkv; a.q = static_cast<uint16_t*>(q_out); a.qkv_stride = qkv_stride; a.q_stride = q_stride;
  a.b = kv_batch_args(b);
  a.c = kv_cache_args(c);
  a.inv_freq = r.inv_freq; a.q_gain = r.q_gain; a.k_gain = r.k_gain; a.eps = r.eps; a.mscale = r.mscale;
  a.heads = heads; a.rot = r.rot_dim; a.inter = r.interleaved;
  const int bt = c.block_tokens, dh = c.head_dim, sl = dh / (bf16 ? 16 : 8), tokens = b.T < bt ? b.T : bt;
  int th = 64;                                   // a thread of the cache part takes 32 values of a head's block
  while (th * 32 < tokens * dh) th *= 2;
  // keys: a work-group goes through several heads, whose angles are the same, where that still leaves two work-groups to a CU (16 prompts of 512 tokens, 32 heads: one head a
  // work-group 103 us, eight 75, as with work-groups for all CUs twice)
  a.seq_blocks = (b.T + bt - 2) / bt + 1;
  const long long blocks = static_cast<long long>(b.S) * a.seq_blocks;
  const long long fewest = (511 + blocks) / blocks;
  a.key_groups = int(fewest < c.n_heads ? fewest : c.n_heads);
  a.group_heads = (c.n_heads + a.key_groups - 1) / a.key_groups;
  a.key_groups = (c.n_heads + a.group_heads - 1) / a.group_heads;
  // query part: as many rows of a sequence side by side as there are, the other lanes take other heads; heads are split until the launch has about
  // four work-groups to a CU
  int rows = 1;
  while (rows < b.T && rows * sl < th) { rows *= 2; ++a.rows_log2; }
  a.row_tiles = (b.T + rows - 1) / rows;
  const int side = th / sl / rows;               // heads side by side in a work-group
  const long long tiles = static_cast<long long>(b.S) * a.row_tiles;
  const long long parts = (1023 + tiles) / tiles;
  const int most = (heads + side - 1) / side;
  a.splits = int(parts < most ? parts : most);
  a.split_heads = (heads + a.splits - 1) / a.splits;
  const long long wgs = blocks * (a.key_groups + c.n_heads) + tiles * a.splits;
  if (wgs * th >= (1ll << 32)) return set_error(MOQE_E_SHAPE, "moqe_kv_append: %lld work-groups", wgs);
  const size_t lds = b.T >= 32 ? size_t(bt) * dh : 0;
  ProfileScope ps(MOQE_PK_OTHER, st);
  const dim3 grid(static_cast<unsigned>(wgs)), block(th);
#define MOQE_APPEND(DH, TH)                                                                    \
  do {                                                                                         \
    if (bf16) hipLaunchKernelGGL((k_kv_append<DH, true, TH>), grid, block, lds, st, a);         \
    else hipLaunchKernelGGL((k_kv_append<DH, false, TH>), grid, block, lds, st, a);             \
  } while (0)
  if (dh == 64) MOQE_APPEND(64, 512);
  else if (dh == 128) MOQE_APPEND(128, 512);
  else if (th <= 512) MOQE_APPEND(256, 512);
  else MOQE_APPEND(256, 1024);
#undef MOQE_APPEND
  return check_launch("kv_append");
}

}  // namespace moqe
