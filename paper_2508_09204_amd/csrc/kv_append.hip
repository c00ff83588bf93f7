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
  int seq_blocks;               // blocks that a sequence of T rows can touch
  int row_tiles, rows_log2;     // query part: tiles of 2^rows_log2 rows of a sequence, ...
  int splits, split_heads;      // ... its heads in parts
};

// A slot is two 8-dim pieces of a head vector that hold whole pairs: (j, j + rot/2) pieces in the half layout, neighbours otherwise.
template <int DH>
__device__ __forceinline__ void slot_dims(const AppendArgs& a, int slot, int* da, int* db) {
  const bool halves = !a.inter && slot * 16 < a.rot;
  *da = halves ? slot * 8 : slot * 16;
  *db = halves ? slot * 8 + a.rot / 2 : slot * 16 + 8;
}

// cos and sin of the slot's eight angles at position p.  They are reduced to a fraction of a turn in 64 bits, where 32 would lose 2^-24 of p * inv_freq; what the
// fraction loses when it is rounded to 32 comes back to first order: without that, keys that lie between two codes took the wrong one more than twice as often.
__device__ __forceinline__ void slot_angles(const AppendArgs& a, int slot, int p, float* cs, float* sn) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    double turns = double(p) * (a.inv_freq[slot * 8 + i] * 0.15915494309189535);
    turns -= rint(turns);
    const float hi = float(turns), lo = float(turns - double(hi)) * 6.2831853f;
    float s, c;
    sincospif(2.f * hi, &s, &c);
    cs[i] = a.mscale * fmaf(-lo, s, c);
    sn[i] = a.mscale * fmaf(lo, c, s);
  }
}

__device__ __forceinline__ void turn(bool inter, const float* cs, const float* sn, float* x) {
  if (inter) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = x[2 * i], v = x[2 * i + 1];
      x[2 * i] = u * cs[i] - v * sn[i];
      x[2 * i + 1] = v * cs[i] + u * sn[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = x[i], v = x[8 + i];
      x[i] = u * cs[i] - v * sn[i];
      x[8 + i] = v * cs[i] + u * sn[i];
    }
  }
}

template <bool BF16> struct Piece;         // eight values as they lie in memory
template <> struct Piece<true> { uint4 q; };
template <> struct Piece<false> { float4 a, b; };
__device__ __forceinline__ void load_piece(const void* base, long long at, Piece<true>* p) {
  p->q = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at);
}
__device__ __forceinline__ void load_piece(const void* base, long long at, Piece<false>* p) {
  const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
  p->a = f[0];
  p->b = f[1];
}
__device__ __forceinline__ void piece_values(const Piece<true>& p, float* x) {
  const uint32_t w[4] = {p.q.x, p.q.y, p.q.z, p.q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void piece_values(const Piece<false>& p, float* x) {
  x[0] = p.a.x; x[1] = p.a.y; x[2] = p.a.z; x[3] = p.a.w; x[4] = p.b.x; x[5] = p.b.y; x[6] = p.b.z; x[7] = p.b.w;
}

// RMS norm of a head vector whose DH / 16 slots lie in neighbouring lanes.
template <int DH>
__device__ __forceinline__ void head_norm(const float* gain, float eps, int da, int db, float* x) {
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) q += x[i] * x[i];
#pragma unroll
  for (int d = 1; d < DH / 16; d *= 2) q += __shfl_xor(q, d);
  const float inv = 1.f / sqrtf(q / float(DH) + eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] *= inv * gain[da + i];
    x[8 + i] *= inv * gain[db + i];
  }
}

__device__ __forceinline__ uint32_t codes4(const float* x, float inv) {      // to nearest even; NaN stays, past 464 gets NaN
  uint32_t w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
}
__device__ __forceinline__ uint32_t rescaled4(uint32_t w, float by) {
  const float x[4] = {__builtin_amdgcn_cvt_f32_fp8(w, 0), __builtin_amdgcn_cvt_f32_fp8(w, 1), __builtin_amdgcn_cvt_f32_fp8(w, 2),
                      __builtin_amdgcn_cvt_f32_fp8(w, 3)};
  return codes4(x, by);
}
// Keys (VALUES false) or values of one block and head: the new tokens lo .. hi of block `blk` of the sequence, which lies in cache block `id`.
template <int DH, bool BF16, bool VALUES>
__device__ __forceinline__ void append_block(const AppendArgs& a, const KvSeq& q, int head, int blk, int id, int lo, int hi, uint8_t* lds, uint32_t* wave_max) {
  constexpr int SL = DH / 16, NS = 2;
  const int bt = 1 << a.c.bt_log2, first = blk << a.c.bt_log2;
  const int slots = (hi - lo) * SL, tid = threadIdx.x, th = blockDim.x;
  const bool held = lo > first;
  const long long bh = static_cast<long long>(id) * a.c.heads + head;
  uint8_t* codes = (VALUES ? a.c.v : a.c.k) + bh * (static_cast<long long>(DH) << a.c.bt_log2);
  float* scale = (VALUES ? a.c.v_scale : a.c.k_scale) + bh;
  const float old = held ? *scale : 0.f;
  const long long col = (a.heads + head + (VALUES ? a.c.heads : 0)) * DH;

  Piece<BF16> pa[NS], pb[NS];
  int da, db;
  slot_dims<DH>(a, tid % SL, &da, &db);
  if (VALUES) { da = tid % SL * 16; db = da + 8; }
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const int u = n * th + tid;
    if (u < slots) {
      const long long at = (q.row0 + (lo + u / SL - q.first())) * a.qkv_stride + col;
      load_piece(a.qkv, at + da, &pa[n]);
      load_piece(a.qkv, at + db, &pb[n]);
    }
  }
  float x[NS][16];
  uint32_t top = 0;
  bool infinite = false;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const int u = n * th + tid;
    if (u < slots) {
      piece_values(pa[n], x[n]);
      piece_values(pb[n], x[n] + 8);
      if (!VALUES) {
        if (a.k_gain) head_norm<DH>(a.k_gain, a.eps, da, db, x[n]);        // whole head vectors are in or out: their slots share u / SL
        if (tid % SL * 16 < a.rot) {
          float cs[8], sn[8];
          slot_angles(a, tid % SL, lo + u / SL, cs, sn);
          turn(a.inter, cs, sn, x[n]);
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t bits = __float_as_uint(x[n][i]) & 0x7fffffffu;
        top = max(top, bits < 0x7f800000u ? bits : 0u);
        infinite |= bits == 0x7f800000u;
      }
    }
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) top = max(top, uint32_t(__shfl_xor(int(top), d)));
  if ((tid & 63) == 0) wave_max[tid >> 6] = top;
  __syncthreads();                               // also: everybody has read the old scale
  for (int w = 0; w < th / 64; ++w) top = max(top, wave_max[w]);
  const float need = __uint_as_float(uint32_t(kv_scale_exponent(top) + 127) << 23);
  const float s = held && !(old < need) ? old : need;
  const float inv = 1.f / s;                     // a power of two: exact
  if (tid == 0) *scale = s;
  if (infinite) {                                // the conversion would make NaN of them
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (fabsf(x[n][i]) == INFINITY) x[n][i] = copysignf(448.f * s, x[n][i]);
  }

  if (held && s > old) {                         // the codes of earlier tokens move to the new scale
    const float by = old * inv;
    for (int u = tid; u < bt * DH / 16; u += th) {
      uint4* p = reinterpret_cast<uint4*>(codes) + u;
      uint4 w = *p;
      uint32_t* d = reinterpret_cast<uint32_t*>(&w);
      if (VALUES) {
        const int t0 = first + u / (2 * DH) * 32 + u % 64 / 16 * 4;               // dword j of a unit: tokens t0 + 16 (j & 1) + 0 .. 3
        if (t0 >= lo) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int left = lo - (t0 + 16 * (j & 1));
          const uint32_t keep = left >= 4 ? 0u : left <= 0 ? ~0u : ~0u << (8 * left);
          d[j] = (rescaled4(d[j], by) & ~keep) | (d[j] & keep);
        }
      } else {
        if (first + u / DH * 16 + u % 16 >= lo) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) d[j] = rescaled4(d[j], by);
      }
      *p = w;
    }
    __syncthreads();                             // before single bytes of the same units are written
  }

  // values of groups of 32 tokens that are new altogether are put in order in LDS, others go byte by byte
  const int g_lo = (lo - first + 31) / 32, g_hi = (hi - first) / 32;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const int u = n * th + tid;
    if (u >= slots) continue;
    const uint32_t w[4] = {codes4(x[n], inv), codes4(x[n] + 4, inv), codes4(x[n] + 8, inv), codes4(x[n] + 12, inv)};
    const uint32_t t = uint32_t(lo - first + u / SL);
    if (VALUES) {
      const bool whole = int(t) / 32 >= g_lo && int(t) / 32 < g_hi;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t at = kv_value_at(t, uint32_t(da + i), DH);
        const uint8_t c = uint8_t(w[i / 4] >> (8 * (i % 4)));
        if (whole) lds[at] = c;
        else codes[at] = c;
      }
    } else {
      *reinterpret_cast<uint2*>(codes + kv_key_at(t, uint32_t(da), DH)) = make_uint2(w[0], w[1]);
      *reinterpret_cast<uint2*>(codes + kv_key_at(t, uint32_t(db), DH)) = make_uint2(w[2], w[3]);
    }
  }
  if (VALUES && g_hi > g_lo) {
    __syncthreads();
    for (int u = g_lo * 2 * DH + tid; u < g_hi * 2 * DH; u += th) reinterpret_cast<uint4*>(codes)[u] = reinterpret_cast<const uint4*>(lds)[u];
  }
}

// Work-groups of the cache part (one for each block a sequence can touch and key head), then of the query part (a row tile and some heads each).
template <int DH, bool BF16>
__global__ __launch_bounds__(1024) void k_kv_append(AppendArgs a) {
  extern __shared__ uint8_t lds[];
  __shared__ uint32_t wave_max[2][16];
  constexpr int SL = DH / 16;
  const int tid = threadIdx.x;
  int w = blockIdx.x;
  const int cache_wgs = a.b.S * a.seq_blocks * a.c.heads;
  if (w < cache_wgs) {
    const int head = w % a.c.heads, s = w / a.c.heads / a.seq_blocks;
    const KvSeq q = kv_seq(a.b, s, a.c.bt_log2);
    const int p0 = max(q.first(), 0), end = min(q.len, q.first() + min(q.n, a.b.T));
    const int blk = (p0 >> a.c.bt_log2) + w / a.c.heads % a.seq_blocks, first = blk << a.c.bt_log2;
    if (first >= end) return;
    const int id = a.b.table[static_cast<long long>(s) * a.b.width + blk];
    if (id < 0 || id >= a.c.n_blocks) return;
    const int lo = max(p0, first), hi = min(end, first + (1 << a.c.bt_log2));
    if (lo >= hi) return;
    append_block<DH, BF16, false>(a, q, head, blk, id, lo, hi, lds, wave_max[0]);
    append_block<DH, BF16, true>(a, q, head, blk, id, lo, hi, lds, wave_max[1]);
    return;
  }
  w -= cache_wgs;
  const int split = w % a.splits, s = w / a.splits / a.row_tiles;
  const int lane_row = (tid / SL) & ((1 << a.rows_log2) - 1), group = tid / SL >> a.rows_log2, groups = blockDim.x / SL >> a.rows_log2;
  const KvSeq q = kv_seq(a.b, s, a.c.bt_log2);
  const int i = (w / a.splits % a.row_tiles << a.rows_log2) + lane_row;
  if (i >= min(q.n, a.b.T)) return;
  int da, db;
  slot_dims<DH>(a, tid % SL, &da, &db);
  const bool turned = tid % SL * 16 < a.rot;
  float cs[8], sn[8];
  if (turned) slot_angles(a, tid % SL, q.first() + i, cs, sn);
  const long long row = static_cast<long long>(q.row0 + i) * a.qkv_stride, to = (q.row0 + i) * a.q_stride;
  const int h_end = min(a.heads, (split + 1) * a.split_heads);
  constexpr int B = BF16 ? 4 : 2;                // heads in flight
  for (int h0 = split * a.split_heads + group; h0 < h_end; h0 += B * groups) {
    Piece<BF16> pa[B], pb[B];
#pragma unroll
    for (int n = 0; n < B; ++n) {
      const int h = h0 + n * groups;
      if (h < h_end) {
        load_piece(a.qkv, row + h * DH + da, &pa[n]);
        load_piece(a.qkv, row + h * DH + db, &pb[n]);
      }
    }
#pragma unroll
    for (int n = 0; n < B; ++n) {
      const int h = h0 + n * groups;
      if (h >= h_end) continue;
      float x[16];
      piece_values(pa[n], x);
      piece_values(pb[n], x + 8);
      if (a.q_gain) head_norm<DH>(a.q_gain, a.eps, da, db, x);
      if (turned) turn(a.inter, cs, sn, x);
      uint32_t o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = kv_pair(x[2 * j], x[2 * j + 1]);
      *reinterpret_cast<uint4*>(a.q + to + h * DH + da) = make_uint4(o[0], o[1], o[2], o[3]);
      *reinterpret_cast<uint4*>(a.q + to + h * DH + db) = make_uint4(o[4], o[5], o[6], o[7]);
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
  const int bt = c.block_tokens, dh = c.head_dim, sl = dh / 16, tokens = b.T < bt ? b.T : bt;
  int th = 64;                                   // a thread takes two slots of a block's new tokens
  while (th * 2 < tokens * sl) th *= 2;
  a.seq_blocks = (b.T + bt - 2) / bt + 1;
  // query part: as many rows of a sequence side by side as there are, the other lanes take other heads; heads are split until the launch has about
  // four work-groups to a CU
  int rows = 1;
  while (rows < b.T && rows * sl < th) { rows *= 2; ++a.rows_log2; }
  a.row_tiles = (b.T + rows - 1) / rows;
  const int side = th / sl / rows;               // heads side by side in a work-group
  const long long tiles = static_cast<long long>(b.S) * a.row_tiles;
  long long parts = (1024 + tiles - 1) / tiles;
  const int most = (heads + side - 1) / side;
  a.splits = int(parts < most ? parts : most);
  a.split_heads = (heads + a.splits - 1) / a.splits;
  const long long wgs = static_cast<long long>(b.S) * a.seq_blocks * c.n_heads + tiles * a.splits;
  if (wgs >= (1ll << 31)) return set_error(MOQE_E_SHAPE, "moqe_kv_append: %lld work-groups", wgs);
  const size_t lds = b.T >= 32 ? size_t(bt) * dh : 0;
  ProfileScope ps(MOQE_PK_OTHER, st);
  const dim3 grid(static_cast<unsigned>(wgs)), block(th);
#define MOQE_APPEND(DH)                                                                        \
  do {                                                                                         \
    if (bf16) hipLaunchKernelGGL((k_kv_append<DH, true>), grid, block, lds, st, a);            \
    else hipLaunchKernelGGL((k_kv_append<DH, false>), grid, block, lds, st, a);                \
  } while (0)
  if (dh == 64) MOQE_APPEND(64);
  else if (dh == 128) MOQE_APPEND(128);
  else MOQE_APPEND(256);
#undef MOQE_APPEND
  return check_launch("kv_append");
}

}  // namespace moqe
