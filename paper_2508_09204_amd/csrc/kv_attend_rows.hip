// Attention over the 8-bit cache for many rows (prompts, chunks of prompts): bound by the matrix cores and by the exponentials beside them.
#include "kv_device.h"

#include <type_traits>

namespace moqe {

// LDS reads issued before this point stay before the matrix products after it: the scheduler would put each read next to its product and wait for it there.
// Other arithmetic may cross.
#define KEEP_READS_AHEAD() __builtin_amdgcn_sched_barrier(0x406)

constexpr int ROWS_W = 4;                  // waves of a work-group (eight: 880 instead of 905 us for 2 x 2048 rows on 16384 tokens, 109 instead of 100 for 16 prompts of 512)

struct RowsArgs {
  const uint16_t* q; uint16_t* out;
  long long q_stride, out_stride;
  KvBatch b; KvCache c; KvScore sc;
  int group, tiles;             // query heads to a key head; column tiles of a sequence and key head at most
  int whole, split_tiles, splits;   // of each XCD's column tiles: so many are done by one work-group each, the tokens of the next are divided into `splits` parts
  KvParts parts;                // [split][split tile][XCD][column of the tile]
};

// Column tile number x of an XCD (work-groups go round robin over 8).  Sequences and key heads are dealt out to the XCDs, all tiles of one to one XCD, whose L2 then holds their
// keys and values; the longest tiles go first.  The tiles of what is left over from eights, in a row, are cut into eight equal stretches: within a head every eighth
// tile comes in turn, so that a stretch that takes a part of a head gets long and short ones.
struct RowsTile { int s, h, tile; };
__device__ __forceinline__ bool rows_tile(const RowsArgs& a, int xcd, int x, RowsTile* t) {
  const int all = a.b.S * a.c.heads, dealt = all / 8 * a.tiles, rest = all % 8 * a.tiles;
  int sh, rank;                                  // rank: from the longest tile of the head on
  if (x < dealt) {
    sh = x / a.tiles * 8 + xcd;
    rank = x % a.tiles;
  } else {
    const int f = static_cast<int>(static_cast<long long>(rest) * xcd / 8) + x - dealt;
    if (f >= static_cast<int>(static_cast<long long>(rest) * (xcd + 1) / 8)) return false;
    const int y = f % a.tiles, n = a.tiles / 8, more = a.tiles % 8 * (n + 1);        // the first tiles % 8 of the eight turns have one more
    sh = all / 8 * 8 + f / a.tiles;
    rank = y < more ? y % (n + 1) * 8 + y / (n + 1) : (y - more) % n * 8 + a.tiles % 8 + (y - more) / n;
  }
  t->s = sh / a.c.heads;
  t->h = sh % a.c.heads;
  t->tile = a.tiles - 1 - rank;
  return true;
}

// One work-group takes 128 columns (row i, query head g of the key head's group: column i * group + g), 32 for each of its four waves, through the tokens in
// tiles of 64.  The tile's codes become bf16 operands once, on their way into LDS (two buffers, one barrier a tile; the codes of the tile after next are already
// under way in registers), in the order in which a wave reads them: 16 bytes a lane in a row, no bank conflicts.  Products are 32 x 32 x 16, half as many
// instructions as 16 x 16 x 32 at the same rate: a SIMD issues them and the softmax's arithmetic through one port, and that port is what it runs out of.
// Scores stay in registers: the layout of S^T = K Q^T is the operand layout of O^T = V^T P^T if 16 tokens of values go 0..3, 8..11 | 4..7, 12..15.
template <int DH, int EXTRA>
__global__ __launch_bounds__(ROWS_W * 64, DH == 256 ? 1 : 2) void k_kv_attend_rows(RowsArgs a) {
  constexpr int W = ROWS_W, COLS = W * 32, KS = DH / 16, DT = DH / 32, U = DH / (W * 16);   // U: 16-byte units of keys (and of values) a thread brings in
  constexpr int HALF = 64 * DH * 2;                                            // bytes of a tile's keys in bf16
  extern __shared__ __align__(16) uint8_t lds[];                               // [2][keys, values]
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, r = lane & 15, kq = lane >> 4, c32 = lane & 31, half = lane >> 5;
  const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  const bool part = slot >= a.whole;
  const int x = part ? a.whole + (slot - a.whole) / a.splits : slot, split = part ? (slot - a.whole) % a.splits : 0, splits = part ? a.splits : 1;
  RowsTile rt;
  if (!rows_tile(a, xcd, x, &rt)) return;
  const int s = rt.s, h = rt.h, tile = rt.tile;
  const KvSeq q = kv_seq(a.b, s, a.c.bt_log2);
  const int rows = min(q.n, a.b.T), first_pos = q.first();
  const int i_first = tile * COLS / a.group;
  if (i_first >= rows) return;
  const int i_last = min((tile * COLS + COLS - 1) / a.group, rows - 1);
  const int p_first = first_pos + i_first, p_last = first_pos + i_last;
  const int pre = a.sc.prefix ? kv_prefix(a.sc.prefix[s], q.len) : 0, window = a.sc.window;
  const int seen = min(q.len, max(max(p_last + 1, pre), 0));                   // tokens from here on are seen by no row of the work-group
  const KvSteps ks = kv_steps(q.len, seen, p_first, window, pre);
  const float scale2 = a.sc.scale2;
  // the wave's own rows, and this lane's: both halves of a wave hold the same 32 columns
  const int col0 = tile * COLS + wave * 32;
  const int w_first = first_pos + min(col0 / a.group, rows - 1), w_last = first_pos + min((col0 + 31) / a.group, rows - 1);
  const bool idle = col0 / a.group >= rows;
  const KvRange wg_all = kv_all_see(p_first, p_last, pre, window), all_see = kv_all_see(w_first, w_last, pre, window),
                some_see = kv_some_see(w_first, w_last, pre, window);
  const int from = max(pre, window > 0 ? w_last - window + 1 : 0);             // steps from here on hide nothing from the wave's rows but what comes after them
  const int col = col0 + c32, row = col / a.group, head = h * a.group + col - row * a.group;
  const bool mine = row < rows;
  const int pos = first_pos + row;
  const KvSight sight = kv_sight(pos, q.len, window);
  const float slope = (EXTRA & KV_BIAS) && mine && a.sc.slopes ? a.sc.slopes[head] * KV_LOG2E : 0.f;

  kv_bf16x8 qf[KS];
  {
    const uint16_t* src = a.q + (q.row0 + row) * a.q_stride + static_cast<long long>(head) * DH + half * 8;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (mine) v = *reinterpret_cast<const uint4*>(src + k * 16);
      qf[k] = __builtin_bit_cast(kv_bf16x8, v);
    }
  }
  kv_f32x16 o[DT];
  float m = -3e38f, l = 0.f;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int y = 0; y < 16; ++y) o[d][y] = 0.f;

  const uint32_t head_bytes = uint32_t(DH) << a.c.bt_log2;
  const int* table = a.b.table + static_cast<long long>(s) * a.b.width;
  const int all_tiles = (ks.count + 1) / 2;
  const int t_begin = static_cast<int>(static_cast<long long>(all_tiles) * split / splits);
  const int t_end = static_cast<int>(static_cast<long long>(all_tiles) * (split + 1) / splits);
  // lane i looks up step `look + i`: block (-1: absent) and scales
  int look = 2 * t_begin, ids = -1;
  float k_scales = 1.f, v_scales = 1.f;
  auto look_up = [&]() {
    ids = -1;
    k_scales = v_scales = 1.f;
    if (look + lane < ks.count) {
      const int id = table[ks.step(look + lane) * 32 >> a.c.bt_log2];
      if (id >= 0 && id < a.c.n_blocks) {
        ids = id;
        k_scales = a.c.k_scale[static_cast<long long>(id) * a.c.heads + h];
        v_scales = a.c.v_scale[static_cast<long long>(id) * a.c.heads + h];
      }
    }
  };
  look_up();
  // A wave's n-th 64 units of a tile: their step, and the place of the first among that step's 2 * DH.
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  constexpr int STEP_U = 2 * DH / 64;                   // waves' worth of units in a step
  auto unit_step = [&](int n) { return STEP_U >= W ? n * W / STEP_U : n * (W / STEP_U) + wave_u / STEP_U; };
  auto unit_place = [&](int n) { return STEP_U >= W ? (n * W % STEP_U + wave_u) * 64 : wave_u % STEP_U * 64; };
  // A tile under way: its codes, and of its two steps the scales and the first token (2^30: absent, seen by nobody; any block's codes do for it).  Two tiles are (one where
  // the head is 256 wide and registers are short): loads have the time of two tiles to come.  2 x 2048 rows on 16384 tokens, one tile / two: 925 / 888 us.
  constexpr int AHEAD = DH == 256 ? 1 : 2;
  struct Staged { uint4 kc[U], vc[U]; float sk[2], sv[2]; int t0[2]; } way[2];
  auto fetch = [&](int t, Staged& g) {
    if (2 * t >= look + 64) { look += 64; look_up(); }
    const uint8_t *kp[2], *vp[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int at = 2 * t + e - look, id = __builtin_amdgcn_readlane(ids, at), first = ks.step(2 * t + e) * 32;
      g.sk[e] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scales), at));
      g.sv[e] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v_scales), at));
      g.t0[e] = id >= 0 ? first : 1 << 30;
      const long long off = static_cast<long long>(max(id, 0) * static_cast<long long>(a.c.heads) + h) * head_bytes + (first & ((1 << a.c.bt_log2) - 1)) * DH;
      kp[e] = a.c.k + off;
      vp[e] = a.c.v + off;
    }
#pragma unroll
    for (int n = 0; n < U; ++n) {
      const uint32_t at = (unit_place(n) + lane) * 16;
      g.kc[n] = *reinterpret_cast<const uint4*>((unit_step(n) ? kp[1] : kp[0]) + at);
      g.vc[n] = *reinterpret_cast<const uint4*>((unit_step(n) ? vp[1] : vp[0]) + at);
    }
  };
  bool nan = false;                    // a value that is NaN lies where some row does not see it and another may
  auto put = [&](int buf, Staged& g) {
    uint8_t* kb = lds + buf * 2 * HALF;
    uint8_t* vb = kb + HALF;
#pragma unroll
    for (int n = 0; n < U; ++n) {
      const int e = unit_step(n), in = unit_place(n);
      const float fk = e ? g.sk[1] : g.sk[0], fv = e ? g.sv[1] : g.sv[0];
      // keys: 16-token tile in / DH, dims 64 * pair + 32 * st + 8 * kq ..: product k = dims / 16, lane (dims / 8 % 2) * 32 + token
      const int a16 = in / DH, pair = in % DH / 64;
      uint8_t* k0 = kb + (e * KS + 4 * pair) * 1024 + kq / 2 * 1024 + ((kq & 1) * 32 + 16 * a16 + r) * 16;
      *reinterpret_cast<kv_bf16x8*>(k0) = kv_operand(g.kc[n].x, g.kc[n].y, fk);
      *reinterpret_cast<kv_bf16x8*>(k0 + 2048) = kv_operand(g.kc[n].z, g.kc[n].w, fk);
      const int t0 = e ? g.t0[1] : g.t0[0];
      if (!wg_all.has(t0)) {
        g.vc[n] = kv_before(g.vc[n], t0 + 4 * kq, seen);
        nan |= __ballot(kv_nan_bytes(g.vc[n]) != 0) != 0;
        g.vc[n] = kv_without_nan(g.vc[n]);
      }
      // values: dims 32 * dpair + 16 * dt + r, tokens 16 * s + 4 * kq ..: product 2 e + s, lane (kq % 2) * 32 + dim, its first or second four tokens
      const int dpair = in / 64;
      uint8_t* v0 = vb + (2 * e * DT + dpair) * 1024 + ((kq & 1) * 32 + r) * 16 + kq / 2 * 8;
      *reinterpret_cast<uint2*>(v0) = kv_four(g.vc[n].x, fv);
      *reinterpret_cast<uint2*>(v0 + DT * 1024) = kv_four(g.vc[n].y, fv);
      *reinterpret_cast<uint2*>(v0 + 256) = kv_four(g.vc[n].z, fv);
      *reinterpret_cast<uint2*>(v0 + DT * 1024 + 256) = kv_four(g.vc[n].w, fv);
    }
  };

  int t0c[2] = {0, 0};
  if (t_begin < t_end) {
    fetch(t_begin, way[0]);
    if (AHEAD == 2 && t_begin + 1 < t_end) fetch(t_begin + 1, way[1]);
    put(0, way[0]);
    t0c[0] = way[0].t0[0]; t0c[1] = way[0].t0[1];
  }
  __builtin_amdgcn_s_waitcnt(0);       // the queries have come: else the loop would wait for all loads under way before its first product, every time
  if (t_begin + AHEAD < t_end) fetch(t_begin + AHEAD, way[0]);
  __syncthreads();
  auto tile_step = [&](int t, auto odd) {
    constexpr int buf = decltype(odd)::value;
    const int t0[2] = {t0c[0], t0c[1]};
    if (t + 1 < t_end) {
      Staged& g = way[AHEAD == 2 ? buf ^ 1 : 0];
      put(buf ^ 1, g);
      t0c[0] = g.t0[0]; t0c[1] = g.t0[1];
      if (t + 1 + AHEAD < t_end) fetch(t + 1 + AHEAD, g);
    }
    const bool some = some_see.has(t0[0]) || some_see.has(t0[1]);
    if (!idle && some) {
      __builtin_amdgcn_s_setprio(1);       // staging steps back for products and softmax: 2 x 2048 rows on 16384 tokens 961 -> 903 us
      const bool full = all_see.has(t0[0]) && all_see.has(t0[1]);
      const uint8_t* kb = lds + buf * 2 * HALF + lane * 16;
      const uint8_t* vb = kb + HALF;
      kv_f32x16 sc[2];
      kv_bf16x8 kf[2][4];
#pragma unroll
      for (int y = 0; y < 4; ++y) kf[0][y] = *reinterpret_cast<const kv_bf16x8*>(kb + (y % 2 * KS + y / 2) * 1024);
#pragma unroll
      for (int n = 0; n < KS / 2; ++n) {                // four of the 2 * KS operands (16 dims, step) at a time, the two steps' sums in turn
        if (n + 1 < KS / 2) {
#pragma unroll
          for (int y = 0; y < 4; ++y) kf[(n + 1) & 1][y] = *reinterpret_cast<const kv_bf16x8*>(kb + (y % 2 * KS + 2 * (n + 1) + y / 2) * 1024);
        }
        KEEP_READS_AHEAD();
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int e = y % 2, k = 2 * n + y / 2;
          if (k == 0) {
#pragma unroll
            for (int z = 0; z < 16; ++z) sc[e][z] = 0.f;
          }
          sc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[n & 1][y], qf[k], sc[e], 0, 0, 0);
        }
      }
      kv_bf16x8 vf[2][4];
#pragma unroll
      for (int d = 0; d < 4; ++d) vf[0][d] = *reinterpret_cast<const kv_bf16x8*>(vb + d * 1024);
      KEEP_READS_AHEAD();
      // score y of step e belongs to token t0[e] + 8 * (y / 4) + 4 * half + y % 4
      if constexpr (EXTRA != KV_PLAIN) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float far = float(pos - t0[e] - 4 * half);
#pragma unroll
          for (int y = 0; y < 16; ++y) sc[e][y] = kv_extra_score<EXTRA>(a.sc, sc[e][y], slope, far - float(y / 4 * 8 + y % 4));
        }
      }
      if (!full) {
        if (t0[0] >= from && t0[1] >= from) {          // only by order
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int last = pos - t0[e] - 4 * half;
#pragma unroll
            for (int y = 0; y < 16; ++y)
              if (y / 4 * 8 + y % 4 > last) sc[e][y] = -INFINITY;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int y = 0; y < 16; ++y)
              if (!sight.sees(t0[e] + y / 4 * 8 + half * 4 + y % 4, pre)) sc[e][y] = -INFINITY;
        }
      }
      float top = sc[0][0];
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int y = 0; y < 16; ++y) top = fmaxf(top, sc[e][y]);
      if (!EXTRA) top *= scale2;
      if (__any(top > m + 8.f)) {          // the running maximum follows only where weights would pass 2^8: the sums are rescaled seldom
        const float mn = fmaxf(m, fmaxf(top, __shfl_xor(top, 32))), f = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= f;
      }
      // Weights rounded to bf16: a second product with what the rounding leaves takes the mean error from 0.0020 to 0.0016 of the outputs and costs 1.14 to 1.43 times the time
      // (2 x 2048 rows on 16384 tokens 904 -> 1227 us), since this kernel is bound by the matrix cores and their issue.
      kv_bf16x8 pf[2][2];
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int y = 0; y < 16; ++y) pf[e][y / 8][y % 8] = static_cast<__bf16>(__builtin_amdgcn_exp2f(EXTRA ? sc[e][y] - m : fmaf(sc[e][y], scale2, -m)));
#pragma unroll
      for (int e = 0; e < 4; ++e) l = kv_add8(pf[e / 2][e % 2], l);
#pragma unroll
      for (int n = 0; n < DT; ++n) {                   // four of the 4 * DT operands (16 tokens, 32 dims) at a time
        if (n + 1 < DT) {
#pragma unroll
          for (int y = 0; y < 4; ++y) vf[(n + 1) & 1][y] = *reinterpret_cast<const kv_bf16x8*>(vb + (4 * (n + 1) + y) * 1024);
        }
        KEEP_READS_AHEAD();
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int g = (4 * n + y) / DT, d = (4 * n + y) % DT;
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[n & 1][y], pf[g / 2][g % 2], o[d], 0, 0, 0);
        }
      }
      __builtin_amdgcn_s_setprio(0);
    }
    __syncthreads();
  };
  for (int t = t_begin; t < t_end; t += 2) {
    tile_step(t, std::integral_constant<int, 0>());
    if (t + 1 < t_end) tile_step(t + 1, std::integral_constant<int, 1>());
  }

  l += __shfl_xor(l, 32);
  const float inv = part ? 1.f : l == 0.f ? 0.f : 1.f / l;
  uint16_t* dst = a.out + (q.row0 + row) * a.out_stride + static_cast<long long>(head) * DH + half * 4;
  const long long at = ((static_cast<long long>(split) * a.split_tiles + x - a.whole) * 8 + xcd) * COLS + wave * 32 + c32;
  float* po = a.parts.o + at * DH + half * 4;
  if (mine) {
    if (part && half == 0) a.parts.ml[at] = make_float2(m, l);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int y = 0; y < 4; ++y) {                    // dims 32 d + 8 y + 4 half ..
        const float v[4] = {o[d][4 * y] * inv, o[d][4 * y + 1] * inv, o[d][4 * y + 2] * inv, o[d][4 * y + 3] * inv};
        if (part) *reinterpret_cast<float4*>(po + d * 32 + y * 8) = make_float4(v[0], v[1], v[2], v[3]);
        else *reinterpret_cast<uint2*>(dst + d * 32 + y * 8) = make_uint2(kv_pair(v[0], v[1]), kv_pair(v[2], v[3]));
      }
  }

  // Values that are NaN and that some rows do not see were left out of the products (0 * NaN would reach everybody): the dims of those who see them become NaN.
  if (__syncthreads_or(nan) == 0) return;
  for (int j = 2 * t_begin; j < min(2 * t_end, ks.count); ++j) {
    const int t0 = ks.step(j) * 32, id = table[t0 >> a.c.bt_log2];
    if (id < 0 || id >= a.c.n_blocks || wg_all.has(t0)) continue;
    const uint8_t* v = a.c.v + (static_cast<long long>(id) * a.c.heads + h) * head_bytes + (t0 & ((1 << a.c.bt_log2) - 1)) * DH;
    for (int tok = 0; tok < 32; ++tok) {
      const bool sees = mine && sight.sees(t0 + tok, pre);
      if (!__any(sees)) continue;
      for (int d = 0; d < DH / 2; ++d) {               // the dims that this lane has written
        const int dim = d / 4 * 8 + half * 4 + d % 4;
        if (sees && (v[kv_value_at(tok, dim, DH)] & 0x7f) == 0x7f) {
          if (part) po[dim - half * 4] = NAN;
          else dst[dim - half * 4] = 0x7fc0;
        }
      }
    }
  }
}

// Joins the parts of the divided tiles: DH / 4 lanes for each column.
template <int DH>
__global__ __launch_bounds__(256) void k_kv_rows_join(RowsArgs a) {
  constexpr int COLS = ROWS_W * 32, L = DH / 4;
  const int c = blockIdx.x * (256 / L) + threadIdx.x / L, lane = threadIdx.x % L;      // column among those of all divided tiles
  const int xcd = c / COLS & 7, ti = c / COLS >> 3;
  RowsTile rt;
  if (ti >= a.split_tiles || !rows_tile(a, xcd, a.whole + ti, &rt)) return;
  const KvSeq q = kv_seq(a.b, rt.s, a.c.bt_log2);
  const int col = rt.tile * COLS + c % COLS, row = col / a.group, head = rt.h * a.group + col - row * a.group;
  if (row >= min(q.n, a.b.T)) return;
  const long long step = static_cast<long long>(a.split_tiles) * 8 * COLS;
  float m = -3e38f, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0; p0 < a.splits; p0 += 4) {           // four parts under way; past the last one the last again, not counted
    float2 x[4];
    float4 v[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const long long at = c + min(p0 + p, a.splits - 1) * step;
      x[p] = a.parts.ml[at];
      v[p] = *reinterpret_cast<const float4*>(a.parts.o + at * DH + lane * 4);
    }
    float mn = m;
#pragma unroll
    for (int p = 0; p < 4; ++p) mn = fmaxf(mn, x[p].x);
    const float old = exp2f(m - mn);
    m = mn;
    l *= old;
    o.x *= old; o.y *= old; o.z *= old; o.w *= old;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      if (p0 + p >= a.splits) break;
      const float f = exp2f(x[p].x - m);
      l += x[p].y * f;
      o.x += f * v[p].x; o.y += f * v[p].y; o.z += f * v[p].z; o.w += f * v[p].w;
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint16_t* dst = a.out + (q.row0 + row) * a.out_stride + static_cast<long long>(head) * DH + lane * 4;
  *reinterpret_cast<uint2*>(dst) = make_uint2(kv_pair(o.x * inv, o.y * inv), kv_pair(o.z * inv, o.w * inv));
}

namespace {
struct RowsPlan { long long tiles, whole, split_tiles, wgs; int splits; };
// An XCD's column tiles (as many as the bounds of the call allow) go over its 32 CUs, two at a time on each.  If 32 or fewer are left over from full rounds of 64, each has
// a CU to itself, or CUs have none, and that takes 0.68 of the time of two side by side: so the tokens of those tiles are divided into as many parts as fill the 64
// places, of at least 512 tokens.  2 x T rows of 7 query heads on 14336 tokens and themselves, tiles an XCD, whole / divided (us): 16 tiles
// 338 / 137, 32 349 / 260, 80 900 / 656, 96 913 / 792.
// More than 32 left over are not divided: 48 tiles 427 / 462, 112 tiles 942 / 968.
RowsPlan rows_plan(const moqe_attention& at, const moqe_kv_batch& b, const moqe_kv_cache& c) {
  constexpr int COLS = ROWS_W * 32, CUS = 32;
  RowsPlan p{};
  p.tiles = (static_cast<long long>(b.T) * (at.n_heads / c.n_heads) + COLS - 1) / COLS;
  const long long heads = static_cast<long long>(b.S) * c.n_heads;
  p.whole = heads / 8 * p.tiles + (heads % 8 * p.tiles + 7) / 8;
  p.splits = 1;
  const long long left = p.whole % (2 * CUS), most = static_cast<long long>(b.table_width) * c.block_tokens / 512;
  if (left > 0 && left <= CUS) {
    const long long k = 2 * CUS / left < most ? 2 * CUS / left : most;
    if (k >= 2) {
      p.splits = static_cast<int>(k < 16 ? k : 16);
      p.split_tiles = left;
      p.whole -= left;
    }
  }
  p.wgs = 8 * (p.whole + p.split_tiles * p.splits);
  return p;
}
size_t rows_parts(const RowsPlan& p) { return size_t(p.splits) * p.split_tiles * 8 * ROWS_W * 32; }
}  // namespace

size_t kv_attend_rows_ws_bytes(const moqe_attention& at, const moqe_kv_batch& b, const moqe_kv_cache& c) {
  const size_t rows = rows_parts(rows_plan(at, b, c));
  return align256(rows * 8) + align256(rows * c.head_dim * 4);
}

int32_t launch_kv_attend_rows(const void* q, long long q_stride, const moqe_attention& at, const moqe_kv_batch& b, const moqe_kv_cache& c,
                              void* out, long long out_stride, void* ws, hipStream_t st) {
  RowsArgs a{};
  a.q = static_cast<const uint16_t*>(q); a.out = static_cast<uint16_t*>(out); a.q_stride = q_stride; a.out_stride = out_stride;
  a.b = kv_batch_args(b);
  a.c = kv_cache_args(c);
  a.sc = kv_score(at, b, c);
  a.group = at.n_heads / c.n_heads;
  const RowsPlan p = rows_plan(at, b, c);
  if (p.wgs >= (1ll << 24)) return set_error(MOQE_E_SHAPE, "moqe_kv_attention: %lld work-groups", p.wgs);
  a.tiles = int(p.tiles);
  a.whole = int(p.whole);
  a.split_tiles = int(p.split_tiles);
  a.splits = p.splits;
  if (p.split_tiles) a.parts = kv_parts(ws, rows_parts(p));
  const int lds = 64 * c.head_dim * 2 * 4;
  const dim3 grid(static_cast<unsigned>(p.wgs)), block(ROWS_W * 64);
  const int extra = kv_extra(at);
  int32_t rc = MOQE_OK;
  ProfileScope ps(MOQE_PK_OTHER, st);
  auto launch = [&](auto dh, auto ex) {
    constexpr int DH = decltype(dh)::value, EX = decltype(ex)::value;
    if (DH == 256) rc = ensure_dynamic_lds(LDSK_ATTEND_ROWS + (EX == KV_FAR_CAP ? 4 : EX), reinterpret_cast<const void*>(k_kv_attend_rows<DH, EX>), lds, "moqe_kv_attention");
    if (!rc) hipLaunchKernelGGL((k_kv_attend_rows<DH, EX>), grid, block, lds, st, a);
  };
  auto launch_dh = [&](auto dh) {
    if (extra == KV_PLAIN) launch(dh, std::integral_constant<int, KV_PLAIN>());
    else if (extra == KV_CAP) launch(dh, std::integral_constant<int, KV_CAP>());
    else if (extra == KV_BIAS) launch(dh, std::integral_constant<int, KV_BIAS>());
    else if (extra == (KV_CAP | KV_BIAS)) launch(dh, std::integral_constant<int, KV_CAP | KV_BIAS>());
    else launch(dh, std::integral_constant<int, KV_FAR_CAP>());
  };
  if (c.head_dim == 64) launch_dh(std::integral_constant<int, 64>());
  else if (c.head_dim == 128) launch_dh(std::integral_constant<int, 128>());
  else launch_dh(std::integral_constant<int, 256>());
  if (rc) return rc;
  if (p.split_tiles) {
    const dim3 jgrid(static_cast<unsigned>(p.split_tiles * 8 * ROWS_W * 32 * (c.head_dim / 4) / 256));
    if (c.head_dim == 64) hipLaunchKernelGGL((k_kv_rows_join<64>), jgrid, dim3(256), 0, st, a);
    else if (c.head_dim == 128) hipLaunchKernelGGL((k_kv_rows_join<128>), jgrid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_kv_rows_join<256>), jgrid, dim3(256), 0, st, a);
  }
  return check_launch("kv_attention");
}

}  // namespace moqe
