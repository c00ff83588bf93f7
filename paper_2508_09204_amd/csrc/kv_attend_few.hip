// Attention over the 8-bit cache for few rows (decode steps, short continuations): bound by reading the cache once.
#include "kv_device.h"

#include <algorithm>
#include <type_traits>

namespace moqe {

struct FewArgs {
  const uint16_t* q; uint16_t* out;
  long long q_stride, out_stride;
  KvBatch b; KvCache c; KvScore sc;
  int group, cols;              // query heads to a key head; columns (rows x group) of a sequence and key head at most
  int target, min_steps;        // chunks wanted in all, steps of 32 tokens that a chunk has at least
  KvParts parts;                // [chunk][key head][column]; NULL: one chunk a sequence
  int2* of_seq;                 // first chunk and chunks of every sequence, for the launch that joins them
};

// How the sequences' steps are cut into chunks, equal ones within a sequence.  Every wave works it out by itself.
struct FewPlan {
  int s, first, chunks, j, j_end;          // sequence, number of its first chunk, its chunks, steps of this one
};
__device__ __forceinline__ KvSteps few_steps(const FewArgs& a, int s, KvSeq* q, int* seen) {
  *q = kv_seq(a.b, s, a.c.bt_log2);
  const int pre = a.sc.prefix ? kv_prefix(a.sc.prefix[s], q->len) : 0, rows = min(q->n, a.b.T);
  *seen = rows > 0 ? min(q->len, max(q->first() + rows, pre)) : 0;             // tokens from here on are seen by no row: nothing of them may be read into a sum
  return kv_steps(q->len, max(*seen, 0), q->first(), a.sc.window, pre);
}
// The sequence that chunk number `w` falls into.  False: there is no such chunk.
__device__ __forceinline__ bool few_plan(const FewArgs& a, int w, FewPlan* p) {
  const int lane = threadIdx.x & 63, S = a.b.S;
  int total = 0;
  for (int base = 0; base < S; base += 64) {
    KvSeq q;
    int seen;
    total += base + lane < S ? few_steps(a, base + lane, &q, &seen).count : 0;
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) total += __shfl_xor(total, d);
  const int steps = max(a.min_steps, (total + a.target - 1) / a.target);
  int before = 0;
  for (int base = 0; base < S; base += 64) {
    KvSeq q;
    int seen;
    const int s = base + lane, count = s < S ? few_steps(a, s, &q, &seen).count : 0;
    const int n = s < S ? max(1, (count + steps - 1) / steps) : 0;
    int upto = n;                                   // inclusive sum over the lanes
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    const unsigned long long hit = __ballot(w < before + upto);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      p->s = base + l;
      p->chunks = __builtin_amdgcn_readlane(n, l);
      p->first = __builtin_amdgcn_readfirstlane(before) + __builtin_amdgcn_readlane(upto, l) - p->chunks;
      const int c = w - p->first, all = __builtin_amdgcn_readlane(count, l);
      const int each = all / p->chunks, more = all - each * p->chunks;        // the first chunks have one step more
      p->j = __builtin_amdgcn_readfirstlane(c * each + min(c, more));
      p->j_end = __builtin_amdgcn_readfirstlane(p->j + each + (c < more ? 1 : 0));
      return true;
    }
    before += __shfl(upto, 63);
  }
  return false;
}

// One work-group takes a chunk of a sequence's tokens for one key head; each of its W waves takes every W-th step of 32 tokens.  A wave reads its step's codes
// straight into matrix-core operands, 16 bytes a lane, and asks for the next step's keys as soon as this one's have gone through their product, for its values
// likewise.  It keeps its own running maximum and sum for the NC * 16 columns (row i, query head g: column i * group + g); the waves' results are joined in LDS.
// Bound by reading the cache: 2 sequences of 131000 tokens, 8 key heads of 128 (537 MB), 98 us, 5.5 TB/s; 64 of up to 8000, 4 key heads (251 MB), 56 us with the join; short ones by
// the trips to memory that wait for one another (lengths, block table, codes): one token on 63 tokens 4.8 us.
// PAIR, up to eight columns: the other eight hold the same queries, hence the same scores, and take what the rounding of the weights to bf16 left, as weights of their own.  One
// product does for both, and the error against 64 bits is that of the rounded result alone (one token on 600: 0.0021 -> 0.0017 of the outputs' size in the mean square, 6.9 -> 7.0 us).  For 9 to 32
// columns that would take a second product, 2 to 7 % of the time: their weights are rounded to bf16, as in the kernel for many rows.
constexpr int FEW_W = 8;
template <int DH, int NC, bool PAIR, int EXTRA>
__global__ __launch_bounds__(FEW_W * 64, NC == 1 && DH <= 128 ? 4 : 1) void k_kv_attend_few(FewArgs a) {
  constexpr int W = FEW_W, KS = DH / 32, DT = DH / 16, KL = DH / 64, VL = DH / 32;
  constexpr int PAD = DH + 4;
  __shared__ float obuf[4][16][PAD];
  __shared__ float2 ml[W][NC * 16];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, r = lane & 15, kq = lane >> 4;
  const int h = blockIdx.x % a.c.heads, w = blockIdx.x / a.c.heads;
  FewPlan pl;
  if (a.parts.o) {
    if (!few_plan(a, w, &pl)) return;
  } else {
    pl = FewPlan{w, w, 1, 0, 1 << 30};
  }
  KvSeq q;
  int seen;
  const KvSteps ks = few_steps(a, pl.s, &q, &seen);
  const int rows = min(q.n, a.b.T), first_pos = q.first();
  if (rows == 0) return;
  const int pre = a.sc.prefix ? kv_prefix(a.sc.prefix[pl.s], q.len) : 0, window = a.sc.window, last_pos = first_pos + rows - 1;
  const KvRange all_see = kv_all_see(first_pos, last_pos, pre, window);
  const int j_begin = pl.j + wave, j_end = min(ks.count, pl.j_end);
  const float scale2 = a.sc.scale2;

  kv_bf16x8 qf[NC][KS];
  KvSight sight[NC];
  int pos[NC];
  float slope[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int col = PAIR ? r & 7 : c * 16 + r, i = col / a.group, g = col - i * a.group;
    const bool in = i < rows;
    pos[c] = first_pos + i;
    sight[c] = kv_sight(pos[c], q.len, window);
    if (EXTRA & KV_BIAS) slope[c] = in && a.sc.slopes ? a.sc.slopes[h * a.group + g] * KV_LOG2E : 0.f;
    const uint16_t* src = a.q + (q.row0 + i) * a.q_stride + static_cast<long long>(h * a.group + g) * DH + kq * 8;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (in) v = *reinterpret_cast<const uint4*>(src + k * 32);
      qf[c][k] = __builtin_bit_cast(kv_bf16x8, v);
    }
  }

  // 64 steps of this wave at a time: lane i looks up step j0 + W i: block (-1: absent, nothing is seen) and scales
  const long long block_bytes = static_cast<long long>(DH) << a.c.bt_log2;
  const int* table = a.b.table + static_cast<long long>(pl.s) * a.b.width;
  int id = -1;
  float k_scale = 0.f, v_scale = 0.f;
  auto look_up = [&](int j0) {
    id = -1;
    const int mine = j0 + W * lane;
    if (mine < j_end) {
      id = table[ks.step(mine) * 32 >> a.c.bt_log2];
      if (id < 0 || id >= a.c.n_blocks) id = -1;
      if (id >= 0) {
        k_scale = a.c.k_scale[static_cast<long long>(id) * a.c.heads + h];
        v_scale = a.c.v_scale[static_cast<long long>(id) * a.c.heads + h];
      }
    }
  };
  uint4 kc[2 * KL], vc[VL];
  auto place = [&](int j, int bid) {
    const int tok = ks.step(j) * 32 & ((1 << a.c.bt_log2) - 1);
    return (static_cast<long long>(bid) * a.c.heads + h) * block_bytes + tok * DH + lane * 16;
  };
  auto load_keys = [&](int j, int bid) {
    const uint8_t* p = a.c.k + place(j, bid);
#pragma unroll
    for (int x = 0; x < 2 * KL; ++x) kc[x] = *reinterpret_cast<const uint4*>(p + x * 1024);
  };
  auto load_values = [&](int j, int bid) {
    const uint8_t* p = a.c.v + place(j, bid);
#pragma unroll
    for (int x = 0; x < VL; ++x) vc[x] = *reinterpret_cast<const uint4*>(p + x * 1024);
  };
  kv_f32x4 o[NC][DT];
  float m[NC], l[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m[c] = -3e38f;
    l[c] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[c][d] = kv_f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const float less = PAIR && r >= 8 ? -1.f : 0.f;
  bool nan = false;
  look_up(j_begin);
  {
    const int bid = max(__builtin_amdgcn_readlane(id, 0), 0);
    load_keys(j_begin, bid);
    load_values(j_begin, bid);
  }
  kv_wait_loads<2 * KL + VL>();          // the queries and scales have come: else the loop would wait for all loads under way before its first product, every time
  int i = 0;                             // the step's place among those looked up
  for (int j = j_begin; j < j_end; j += W) {
    const int bid = __builtin_amdgcn_readlane(id, i);
    const float sk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scale), i));
    const float sv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v_scale), i));
    // the next step's block; where there is none, any block does: nothing of it is seen
    int next = max(bid, 0);
    i = (i + 1) & 63;
    if (j + W < j_end) {
      if (i == 0) look_up(j + W);
      next = max(__builtin_amdgcn_readlane(id, i), 0);
    }
    const int t0 = bid < 0 ? 1 << 30 : ks.step(j) * 32;
    const bool full = all_see.has(t0);
    kv_f32x4 s[2][NC];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int c = 0; c < NC; ++c) s[t][c] = kv_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const uint4 u = kc[t * KL + k / 2];
        const kv_bf16x8 kf = (k & 1) ? kv_operand(u.z, u.w, sk) : kv_operand(u.x, u.y, sk);
#pragma unroll
        for (int c = 0; c < NC; ++c) s[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[c][k], s[t][c], 0, 0, 0);
        if (k % 2) __builtin_amdgcn_sched_barrier(0);       // else all operands are converted ahead of all products, and the registers do not hold them
      }
    }
    load_keys(j + W, next);
    kv_bf16x8 pf[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float top = -INFINITY;
      const float far = float(pos[c] - t0 - 4 * kq);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int tok = t0 + 16 * t + 4 * kq + x;
          if constexpr (EXTRA != KV_PLAIN) s[t][c][x] = kv_extra_score<EXTRA>(a.sc, s[t][c][x], slope[c], far - float(16 * t + x));
          if (!full && !sight[c].sees(tok, pre)) s[t][c][x] = -INFINITY;
          top = fmaxf(top, s[t][c][x]);
        }
      if (!EXTRA) top *= scale2;
      if (__any(top > m[c] + 8.f)) {       // the running maximum follows only where weights would pass 2^8: the sums are rescaled seldom
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m[c], top), f = __builtin_amdgcn_exp2f(m[c] - mn);
        m[c] = mn;
        l[c] *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[c][d] *= f;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float weight = __builtin_amdgcn_exp2f(EXTRA ? s[t][c][x] - m[c] : fmaf(s[t][c][x], scale2, -m[c]));
          pf[c][4 * t + x] = static_cast<__bf16>(PAIR ? fmaf(less, static_cast<float>(static_cast<__bf16>(weight)), weight) : weight);
        }
      l[c] = kv_add8(pf[c], l[c]);
    }
    if (!full) {                         // values that are NaN must not reach rows that do not see them: 0 * NaN would
#pragma unroll
      for (int x = 0; x < VL; ++x) {
        vc[x] = kv_before(vc[x], t0 + 4 * kq, seen);
        nan |= __ballot(kv_nan_bytes(vc[x]) != 0) != 0;
        vc[x] = kv_without_nan(vc[x]);
      }
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const uint4 u = vc[d / 2];
      const kv_bf16x8 vf = (d & 1) ? kv_operand(u.z, u.w, sv) : kv_operand(u.x, u.y, sv);
#pragma unroll
      for (int c = 0; c < NC; ++c) o[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[c], o[c][d], 0, 0, 0);
      if (d % 2) __builtin_amdgcn_sched_barrier(0);
    }
    load_values(j + W, next);
  }

  if (a.parts.o && w == pl.first && h == 0 && tid == 0) a.of_seq[pl.s] = make_int2(pl.first, pl.chunks);      // not earlier: loads after a store are not scalar
  // the waves' results: common maximum, then sums in a fixed order: wave v + 4 joins wave v, then four waves in a row
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] += __shfl_xor(l[c], 16);
    l[c] += __shfl_xor(l[c], 32);
    if (PAIR) l[c] += __shfl_xor(l[c], 8);
    if (kq == 0) ml[wave][c * 16 + r] = make_float2(m[c], l[c]);
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float mt = ml[0][c * 16 + r].x;
#pragma unroll
    for (int v = 1; v < W; ++v) mt = fmaxf(mt, ml[v][c * 16 + r].x);
    const float f = exp2f(m[c] - mt);
    if (c > 0) __syncthreads();              // the columns before have been read
    if (wave >= 4) {
#pragma unroll
      for (int d = 0; d < DT; ++d) *reinterpret_cast<kv_f32x4*>(&obuf[wave & 3][r][d * 16 + kq * 4]) = o[c][d] * f;
    }
    __syncthreads();
    if (wave < 4) {                          // a lane reads and writes its own places
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        kv_f32x4* at = reinterpret_cast<kv_f32x4*>(&obuf[wave][r][d * 16 + kq * 4]);
        *at += o[c][d] * f;
      }
    }
    __syncthreads();
    constexpr int V = DH / (W * 4);          // values a thread gathers
    const int oc = tid / (W * 4), col = c * 16 + oc, d0 = tid % (W * 4) * V, row = col / a.group, g = col - row * a.group;
    if (row < rows) {
      float mm = ml[0][col].x, lt = 0.f;
#pragma unroll
      for (int v = 1; v < W; ++v) mm = fmaxf(mm, ml[v][col].x);
#pragma unroll
      for (int v = 0; v < W; ++v) lt += ml[v][col].y * exp2f(ml[v][col].x - mm);
      float y[V];
#pragma unroll
      for (int e = 0; e < V; ++e) y[e] = ((obuf[0][oc][d0 + e] + obuf[1][oc][d0 + e]) + obuf[2][oc][d0 + e]) + obuf[3][oc][d0 + e];
      if (PAIR) {                              // row < rows: oc is below 8
#pragma unroll
        for (int e = 0; e < V; ++e)
          y[e] += ((obuf[0][oc + 8][d0 + e] + obuf[1][oc + 8][d0 + e]) + obuf[2][oc + 8][d0 + e]) + obuf[3][oc + 8][d0 + e];
      }
      if (pl.chunks == 1) {
        const float inv = lt == 0.f ? 0.f : 1.f / lt;
        uint16_t* dst = a.out + (q.row0 + row) * a.out_stride + static_cast<long long>(h * a.group + g) * DH + d0;
#pragma unroll
        for (int e = 0; e < V; e += 2) *reinterpret_cast<uint32_t*>(dst + e) = kv_pair(y[e] * inv, y[e + 1] * inv);
      } else {
        const long long at = (static_cast<long long>(w) * a.c.heads + h) * a.cols + col;
        if (d0 == 0) a.parts.ml[at] = make_float2(mm, lt);
#pragma unroll
        for (int e = 0; e < V; ++e) a.parts.o[at * DH + d0 + e] = y[e];
      }
    }
  }

  // NaN among values that some rows do not see was left out of the products: the dims of those who see it become NaN
  if (__syncthreads_or(nan) == 0 || !nan) return;
  for (int j = j_begin; j < j_end; j += W) {
    const int t0 = ks.step(j) * 32, bid = table[t0 >> a.c.bt_log2];
    if (bid < 0 || bid >= a.c.n_blocks || all_see.has(t0)) continue;
    const uint8_t* v = a.c.v + (static_cast<long long>(bid) * a.c.heads + h) * block_bytes + (t0 & ((1 << a.c.bt_log2) - 1)) * DH + lane * 16;
#pragma unroll 1
    for (int d = 0; d < DT; ++d) {
      const uint2 w2 = *reinterpret_cast<const uint2*>(v + d / 2 * 1024 + d % 2 * 8);
      const kv_bf16x8 bad = kv_operand(kv_nan_bytes(w2.x) * 0x38u, kv_nan_bytes(w2.y) * 0x38u, 1.f);    // 1 where the code is NaN
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        kv_bf16x8 sees;
#pragma unroll
        for (int y = 0; y < 8; ++y) sees[y] = static_cast<__bf16>(sight[c].sees(t0 + y / 4 * 16 + 4 * kq + y % 4, pre) ? 1.f : 0.f);
        const kv_f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad, sees, kv_f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
        const int col = c * 16 + r, row = col / a.group, g = col - row * a.group;
        if (row >= rows) continue;
#pragma unroll
        for (int y = 0; y < 4; ++y)
          if (n[y] > 0.f) {
            const int dim = d * 16 + kq * 4 + y;
            if (pl.chunks == 1) a.out[(q.row0 + row) * a.out_stride + static_cast<long long>(h * a.group + g) * DH + dim] = 0x7fc0;
            else a.parts.o[((static_cast<long long>(w) * a.c.heads + h) * a.cols + col) * DH + dim] = NAN;
          }
      }
    }
  }
}

// Joins the chunks: a work-group for each column of a sequence and key head.  DH / 4 lanes hold a row; the 1024 / DH such groups of lanes take every so many-th
// chunk, and their sums are added in order.  The first chunk of each group is asked for along with the maxima.
template <int DH>
__global__ __launch_bounds__(256) void k_kv_attend_join(FewArgs a) {
  constexpr int L = DH / 4, GROUPS = 256 / L;
  __shared__ float4 sums[GROUPS][L];
  __shared__ float lsum[GROUPS];
  const int group = threadIdx.x / L, lane = threadIdx.x % L;
  const int h = blockIdx.x % a.c.heads, s = blockIdx.x / a.c.heads / a.cols, col = blockIdx.x / a.c.heads % a.cols;
  const int2 of_seq = a.of_seq[s];
  const KvSeq q = kv_seq(a.b, s, a.c.bt_log2);
  const int chunks = of_seq.y, i = col / a.group, g = col - i * a.group;
  if (chunks <= 1 || i >= min(q.n, a.b.T)) return;
  const long long step = static_cast<long long>(a.c.heads) * a.cols, at = of_seq.x * step + static_cast<long long>(h) * a.cols + col;
  float2 x = make_float2(-3e38f, 0.f);
  float4 p = make_float4(0.f, 0.f, 0.f, 0.f);
  auto load = [&](int c) {
    x = a.parts.ml[at + c * step];
    p = *reinterpret_cast<const float4*>(a.parts.o + (at + c * step) * DH + lane * 4);
  };
  if (group < chunks) load(group);
  float m = -3e38f;
  for (int c = threadIdx.x & 63; c < chunks; c += 64) m = fmaxf(m, a.parts.ml[at + c * step].x);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  float f = exp2f(x.x - m), l = x.y * f;
  float4 o = make_float4(f * p.x, f * p.y, f * p.z, f * p.w);
#pragma unroll 8
  for (int c = group + GROUPS; c < chunks; c += GROUPS) {
    load(c);
    f = exp2f(x.x - m);
    l += x.y * f;
    o.x += f * p.x; o.y += f * p.y; o.z += f * p.z; o.w += f * p.w;
  }
  sums[group][lane] = o;
  if (lane == 0) lsum[group] = l;
  __syncthreads();
  if (group > 0) return;
#pragma unroll
  for (int v = 1; v < GROUPS; ++v) {
    const float4 y = sums[v][lane];
    o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
    l += lsum[v];
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint16_t* dst = a.out + (q.row0 + i) * a.out_stride + static_cast<long long>(h * a.group + g) * DH + lane * 4;
  *reinterpret_cast<uint2*>(dst) = make_uint2(kv_pair(o.x * inv, o.y * inv), kv_pair(o.z * inv, o.w * inv));
}

namespace {
// Chunks wanted of a key head: as many work-groups as run at once (two a CU; one where the head is wide or there are more than 16 columns), or the smallest multiple of that
// with one for each sequence, less the half chunk that each sequence adds by rounding up.  Chunks of fewer than 32 steps, four a wave, are mostly the time of their first loads.
// One round / 1024 / 2048 work-groups wanted: 2 sequences of 131000 tokens 98 / 103 / 120 us, 64 of up to 8000 57 / 58 / 65.
constexpr int FEW_MIN_STEPS = 32;
int few_target(const moqe_kv_batch& b, const moqe_kv_cache& c, int cols) {
  const int at_once = cols <= 16 && c.head_dim <= 128 ? 512 : 256;
  const long long round = at_once / c.n_heads > 0 ? at_once / c.n_heads : 1, rounds = (b.S + round - 1) / round;
  return static_cast<int>(rounds * round - b.S / 2);
}
// One chunk a sequence where none can have more than 64 steps, by the table or by the window: eight steps a wave take no longer than half of them and the join.  One / two chunks:
// one sequence of 2000 tokens 8.4 / 10.8 us, 64 of 1400 17 / 26, 96 of 1900 54 / 62; of 3000 (94 steps) 15.1 / 12.7.
constexpr int FEW_ONE_CHUNK = 64;
bool few_one_chunk(const moqe_attention& at, const moqe_kv_batch& b, const moqe_kv_cache& c) {
  long long most = static_cast<long long>(b.table_width) * c.block_tokens / 32;
  if (at.window > 0 && !at.prefix) most = std::min(most, (static_cast<long long>(at.window) + b.T + 30) / 32 + 1);
  return most <= FEW_ONE_CHUNK;
}
// Chunks at most that the workspace holds parts of; 0 where a table has no more than 32 steps (from there on the workspace does not depend on how a call is divided).
long long few_chunks(const moqe_kv_batch& b, const moqe_kv_cache& c, int cols) {
  if (static_cast<long long>(b.table_width) * c.block_tokens / 32 <= FEW_MIN_STEPS) return 0;
  return few_target(b, c, cols) + static_cast<long long>(b.S);
}
}  // namespace

size_t kv_attend_few_ws_bytes(const moqe_attention& at, const moqe_kv_batch& b, const moqe_kv_cache& c) {
  const int cols = b.T * (at.n_heads / c.n_heads);
  const size_t rows = size_t(few_chunks(b, c, cols)) * c.n_heads * cols;
  return align256(rows * 8) + align256(rows * c.head_dim * 4) + align256(rows ? size_t(b.S) * 8 : 0);
}

int32_t launch_kv_attend_few(const void* q, long long q_stride, const moqe_attention& at, const moqe_kv_batch& b, const moqe_kv_cache& c,
                             void* out, long long out_stride, void* ws, hipStream_t st) {
  FewArgs a{};
  a.q = static_cast<const uint16_t*>(q); a.out = static_cast<uint16_t*>(out); a.q_stride = q_stride; a.out_stride = out_stride;
  a.b = kv_batch_args(b);
  a.c = kv_cache_args(c);
  a.sc = kv_score(at, b, c);
  a.group = at.n_heads / c.n_heads;
  a.cols = b.T * a.group;
  a.target = few_target(b, c, a.cols);
  a.min_steps = FEW_MIN_STEPS;
  const long long chunks = few_one_chunk(at, b, c) ? 0 : few_chunks(b, c, a.cols);
  if (chunks) {
    const size_t rows = size_t(chunks) * c.n_heads * a.cols;
    a.parts = kv_parts(ws, rows);
    a.of_seq = reinterpret_cast<int2*>(static_cast<uint8_t*>(ws) + align256(rows * 8) + align256(rows * c.head_dim * 4));
  }
  const long long wgs = (chunks ? chunks : b.S) * c.n_heads;
  const long long join_wgs = chunks ? static_cast<long long>(b.S) * c.n_heads * a.cols : 0;
  if (wgs >= (1ll << 23) || join_wgs >= (1ll << 24)) return set_error(MOQE_E_SHAPE, "moqe_kv_attention: %lld and %lld work-groups", wgs, join_wgs);
  ProfileScope ps(MOQE_PK_OTHER, st);
  const dim3 grid(static_cast<unsigned>(wgs));
  const int extra = kv_extra(at);
  auto launch = [&](auto dh, auto cols, auto pair) {
    constexpr int DH = decltype(dh)::value, NC = decltype(cols)::value;
    constexpr bool PAIR = decltype(pair)::value;
    const dim3 block(FEW_W * 64);
    if (extra == KV_PLAIN) hipLaunchKernelGGL((k_kv_attend_few<DH, NC, PAIR, KV_PLAIN>), grid, block, 0, st, a);
    else if (extra == KV_CAP) hipLaunchKernelGGL((k_kv_attend_few<DH, NC, PAIR, KV_CAP>), grid, block, 0, st, a);
    else if (extra == KV_BIAS) hipLaunchKernelGGL((k_kv_attend_few<DH, NC, PAIR, KV_BIAS>), grid, block, 0, st, a);
    else if (extra == (KV_CAP | KV_BIAS)) hipLaunchKernelGGL((k_kv_attend_few<DH, NC, PAIR, KV_CAP | KV_BIAS>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_kv_attend_few<DH, NC, PAIR, KV_FAR_CAP>), grid, block, 0, st, a);
  };
  auto launch_cols = [&](auto dh) {
    if constexpr (decltype(dh)::value < 256) {
      if (a.cols > 16) return launch(dh, std::integral_constant<int, 2>(), std::false_type());
    }
    if (a.cols > 8) launch(dh, std::integral_constant<int, 1>(), std::false_type());
    else launch(dh, std::integral_constant<int, 1>(), std::true_type());
  };
  if (c.head_dim == 64) launch_cols(std::integral_constant<int, 64>());
  else if (c.head_dim == 128) launch_cols(std::integral_constant<int, 128>());
  else launch_cols(std::integral_constant<int, 256>());
  if (chunks) {
    const dim3 jgrid(static_cast<unsigned>(join_wgs));
    if (c.head_dim == 64) hipLaunchKernelGGL((k_kv_attend_join<64>), jgrid, dim3(256), 0, st, a);
    else if (c.head_dim == 128) hipLaunchKernelGGL((k_kv_attend_join<128>), jgrid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_kv_attend_join<256>), jgrid, dim3(256), 0, st, a);
  }
  return check_launch("kv_attention");
}

}  // namespace moqe
