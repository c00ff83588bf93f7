// Attention over the 8-bit cache for many rows (prompts, chunks of prompts): bound by the matrix cores and by the exponentials beside them.
#include "kv_device.h"

namespace moqe {

struct RowsArgs {
  const uint16_t* q; uint16_t* out;
  long long q_stride, out_stride;
  KvBatch b; KvCache c; KvScore sc;
  int group, tiles, cols;       // query heads to a key head; column tiles, and columns, of a sequence and key head at most
  int splits;                   // parts that the tokens of every column tile are divided into
  KvParts parts;                // [split][sequence][key head][column]
};

// One work-group takes 128 columns (row i, query head g of the key head's group: column i * group + g), 32 for each of its four waves (64 and 16 where the head
// is 256 wide: more does not fit the registers), through the
// tokens in tiles of 64.  The tile's codes become bf16 operands once, on their way into LDS (two buffers, one barrier a tile; the codes of the tile after
// next are already under way in registers), in the order in which a wave reads them: 16 bytes a lane in a row, no bank conflicts.  Scores stay in registers:
// the layout of S^T = K Q^T is the operand layout of O^T = V^T P^T.
// EXTRA: scores are capped, biased, or their scale is not positive.
template <int DH, bool EXTRA>
__global__ __launch_bounds__(256, 2) void k_kv_attend_rows(RowsArgs a) {
  constexpr int NC = DH == 256 ? 1 : 2, COLS = NC * 64, KS = DH / 32, DT = DH / 16, U = DH / 64;   // U: 16-byte units of keys (and of values) a thread brings in
  constexpr int HALF = 64 * DH * 2;                                            // bytes of a tile's keys in bf16
  extern __shared__ __align__(16) uint8_t lds[];                               // [2][keys, values]
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, r = lane & 15, kq = lane >> 4;
  // work-groups of one sequence and key head stay on one XCD (round robin over 8): its L2 holds their keys and values; the longest tiles go first
  const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  const int per = a.tiles * a.splits, sh = slot / per * 8 + xcd;
  if (sh >= a.b.S * a.c.heads) return;
  const int h = sh % a.c.heads, s = sh / a.c.heads, split = slot % a.splits, tile = a.tiles - 1 - slot % per / a.splits;
  const KvSeq q = kv_seq(a.b, s, a.c.bt_log2);
  const int rows = min(q.n, a.b.T), first_pos = q.first();
  const int i_first = tile * COLS / a.group;
  if (i_first >= rows) return;
  const int i_last = min((tile * COLS + COLS - 1) / a.group, rows - 1);
  const int p_first = first_pos + i_first, p_last = first_pos + i_last;
  const int pre = a.sc.prefix ? min(a.sc.prefix[s], q.len) : 0, window = a.sc.window;
  const KvSteps ks = kv_steps(q.len, min(q.len, max(max(p_last + 1, pre), 0)), p_first, window, pre);
  const float scale2 = a.sc.scale * KV_LOG2E;
  // the wave's own rows
  const int col0 = tile * COLS + wave * NC * 16;
  const int w_first = first_pos + min(col0 / a.group, rows - 1), w_last = first_pos + min((col0 + NC * 16 - 1) / a.group, rows - 1);
  const bool idle = col0 / a.group >= rows;

  kv_bf16x8 qf[NC][KS];
  KvSight sight[NC];
  int pos[NC];
  float slope[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int col = col0 + c * 16 + r, i = col / a.group, g = col - i * a.group;
    const bool in = i < rows;
    pos[c] = first_pos + i;
    sight[c] = kv_sight(pos[c], q.len, window);
    if (EXTRA) slope[c] = in && a.sc.slopes ? a.sc.slopes[h * a.group + g] * KV_LOG2E : 0.f;
    const uint16_t* src = a.q + (q.row0 + i) * a.q_stride + static_cast<long long>(h * a.group + g) * DH + kq * 8;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (in) v = *reinterpret_cast<const uint4*>(src + k * 32);
      qf[c][k] = __builtin_bit_cast(kv_bf16x8, v);
    }
  }
  kv_f32x4 o[NC][DT];
  float m[NC], l[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m[c] = -3e38f;
    l[c] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[c][d] = kv_f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const long long block_bytes = static_cast<long long>(DH) << a.c.bt_log2;
  const int* table = a.b.table + static_cast<long long>(s) * a.b.width;
  const int all_tiles = (ks.count + 1) / 2;
  const int t_begin = static_cast<int>(static_cast<long long>(all_tiles) * split / a.splits);
  const int t_end = static_cast<int>(static_cast<long long>(all_tiles) * (split + 1) / a.splits);
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
  // The tile under way: its codes, and of its two steps the scales and the first token (2^30: absent, seen by nobody).
  uint4 kc[U], vc[U];
  float sk[2], sv[2];
  int t0n[2];
  auto fetch = [&](int t) {
    if (2 * t >= look + 64) { look += 64; look_up(); }
    int id[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      id[e] = __builtin_amdgcn_readlane(ids, 2 * t + e - look);
      sk[e] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scales), 2 * t + e - look));
      sv[e] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v_scales), 2 * t + e - look));
      t0n[e] = id[e] >= 0 ? ks.step(2 * t + e) * 32 : 1 << 30;
    }
#pragma unroll
    for (int n = 0; n < U; ++n) {
      const int u = n * 256 + tid, e = __builtin_amdgcn_readfirstlane(n * 256 + (tid & ~63)) / (2 * DH);    // the step of this wave's units
      const int bid = e ? id[1] : id[0];
      kc[n] = vc[n] = make_uint4(0, 0, 0, 0);
      if (bid >= 0) {
        const int tok = (e ? t0n[1] : t0n[0]) & ((1 << a.c.bt_log2) - 1);
        const long long at = (static_cast<long long>(bid) * a.c.heads + h) * block_bytes + tok * DH + (u % (2 * DH)) * 16;
        kc[n] = *reinterpret_cast<const uint4*>(a.c.k + at);
        vc[n] = *reinterpret_cast<const uint4*>(a.c.v + at);
      }
    }
  };
  bool nan = false;                    // a value that is NaN lies where some row does not see it
  auto put = [&](int buf) {
    uint8_t* kb = lds + buf * 2 * HALF;
    uint8_t* vb = kb + HALF;
#pragma unroll
    for (int n = 0; n < U; ++n) {
      const int u = n * 256 + tid, e = __builtin_amdgcn_readfirstlane(n * 256 + (tid & ~63)) / (2 * DH);
      const float fk = e ? sk[1] : sk[0], fv = e ? sv[1] : sv[0];
      const int at = (u >> 6) * 2048 + lane * 16;           // a unit is two operands, 1 KB apart
      *reinterpret_cast<kv_bf16x8*>(kb + at) = kv_operand(kc[n].x, kc[n].y, fk);
      *reinterpret_cast<kv_bf16x8*>(kb + at + 1024) = kv_operand(kc[n].z, kc[n].w, fk);
      if (!kv_all_see(e ? t0n[1] : t0n[0], p_first, p_last, pre, window)) {
        nan |= __ballot(kv_nan_bytes(vc[n]) != 0) != 0;
        vc[n] = kv_without_nan(vc[n]);
      }
      *reinterpret_cast<kv_bf16x8*>(vb + at) = kv_operand(vc[n].x, vc[n].y, fv);
      *reinterpret_cast<kv_bf16x8*>(vb + at + 1024) = kv_operand(vc[n].z, vc[n].w, fv);
    }
  };

  int t0c[2] = {0, 0};
  if (t_begin < t_end) {
    fetch(t_begin);
    put(0);
    t0c[0] = t0n[0]; t0c[1] = t0n[1];
    if (t_begin + 1 < t_end) fetch(t_begin + 1);
  }
  __syncthreads();
  for (int t = t_begin; t < t_end; ++t) {
    const int buf = (t - t_begin) & 1;
    const int t0[2] = {t0c[0], t0c[1]};
    if (t + 1 < t_end) {
      put(buf ^ 1);
      t0c[0] = t0n[0]; t0c[1] = t0n[1];
      if (t + 2 < t_end) fetch(t + 2);
    }
    const bool some = kv_some_see(t0[0], w_first, w_last, pre, window) || kv_some_see(t0[1], w_first, w_last, pre, window);
    if (!idle && some) {
      const bool full = kv_all_see(t0[0], w_first, w_last, pre, window) && kv_all_see(t0[1], w_first, w_last, pre, window);
      const uint8_t* kb = lds + buf * 2 * HALF + lane * 16;
      const uint8_t* vb = kb + HALF;
      kv_f32x4 sc[4][NC];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
#pragma unroll
        for (int c = 0; c < NC; ++c) sc[x][c] = kv_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const kv_bf16x8 kf = *reinterpret_cast<const kv_bf16x8*>(kb + (x * KS + k) * 1024);
#pragma unroll
          for (int c = 0; c < NC; ++c) sc[x][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[c][k], sc[x][c], 0, 0, 0);
        }
      }
      kv_bf16x8 pf[NC][2];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (EXTRA) {
#pragma unroll
          for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              float v = sc[x][c][y];
              v = a.sc.cap > 0.f ? kv_capped(v * a.sc.scale, a.sc.cap) * KV_LOG2E : v * scale2;
              sc[x][c][y] = v - slope[c] * fabsf(float(pos[c] - (t0[x / 2] + 16 * (x & 1) + 4 * kq + y)));
            }
        }
        if (!full) {
#pragma unroll
          for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y)
              if (!sight[c].sees(t0[x / 2] + 16 * (x & 1) + 4 * kq + y, pre)) sc[x][c][y] = -INFINITY;
        }
        float top = sc[0][c][0];
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int y = 0; y < 4; ++y) top = fmaxf(top, sc[x][c][y]);
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
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const float e = __builtin_amdgcn_exp2f(EXTRA ? sc[x][c][y] - m[c] : fmaf(sc[x][c][y], scale2, -m[c]));
            l[c] += e;
            pf[c][x / 2][4 * (x & 1) + y] = static_cast<__bf16>(e);
          }
      }
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const kv_bf16x8 vf = *reinterpret_cast<const kv_bf16x8*>(vb + (g * DT + d) * 1024);
#pragma unroll
          for (int c = 0; c < NC; ++c) o[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[c][g], o[c][d], 0, 0, 0);
        }
    }
    __syncthreads();
  }

  const bool part = a.splits > 1;
  float* po[NC];
  uint16_t* dst[NC];
  bool mine[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] += __shfl_xor(l[c], 16);
    l[c] += __shfl_xor(l[c], 32);
    const float inv = part ? 1.f : l[c] == 0.f ? 0.f : 1.f / l[c];
    const int col = col0 + c * 16 + r, i = col / a.group, g = col - i * a.group;
    mine[c] = i < rows;
    dst[c] = a.out + (q.row0 + i) * a.out_stride + static_cast<long long>(h * a.group + g) * DH + kq * 4;
    const long long at = ((static_cast<long long>(split) * a.b.S + s) * a.c.heads + h) * a.cols + col;
    po[c] = a.parts.o + at * DH + kq * 4;
    if (!mine[c]) continue;
    if (part && kq == 0) a.parts.ml[at] = make_float2(m[c], l[c]);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const kv_f32x4 v = o[c][d] * inv;
      if (part) {
        *reinterpret_cast<kv_f32x4*>(po[c] + d * 16) = v;
      } else {
        uint32_t w[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) w[y] = kv_pair(v[2 * y], v[2 * y + 1]);
        *reinterpret_cast<uint2*>(dst[c] + d * 16) = make_uint2(w[0], w[1]);
      }
    }
  }

  // Values that are NaN and that some rows do not see were left out of the products (0 * NaN would reach everybody): the dims of those who see them become NaN.
  if (__syncthreads_or(nan) == 0) return;
  for (int j = 2 * t_begin; j < min(2 * t_end, ks.count); ++j) {
    const int t0 = ks.step(j) * 32, id = table[t0 >> a.c.bt_log2];
    if (id < 0 || id >= a.c.n_blocks || kv_all_see(t0, p_first, p_last, pre, window)) continue;
    const uint8_t* v = a.c.v + (static_cast<long long>(id) * a.c.heads + h) * block_bytes + (t0 & ((1 << a.c.bt_log2) - 1)) * DH + lane * 16;
#pragma unroll 1
    for (int d = 0; d < DT; ++d) {
      const uint2 w = *reinterpret_cast<const uint2*>(v + d / 2 * 1024 + d % 2 * 8);
      const kv_bf16x8 bad = kv_operand(kv_nan_bytes(w.x) * 0x38u, kv_nan_bytes(w.y) * 0x38u, 1.f);      // 1 where the code is NaN
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        kv_bf16x8 sees;
#pragma unroll
        for (int y = 0; y < 8; ++y) sees[y] = static_cast<__bf16>(sight[c].sees(t0 + y / 4 * 16 + 4 * kq + y % 4, pre) ? 1.f : 0.f);
        const kv_f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad, sees, kv_f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
        for (int y = 0; y < 4; ++y)
          if (mine[c] && n[y] > 0.f) {
            if (part) po[c][d * 16 + y] = NAN;
            else dst[c][d * 16 + y] = 0x7fc0;
          }
      }
    }
  }
}

namespace {
int rows_cols(int dh) { return dh == 256 ? 64 : 128; }
struct RowsPlan { long long tiles, wgs; int splits; };
// Work-groups of a column tile each; where they are less than two to a CU (the bounds of the call say so), its tokens are divided, down to 1024 tokens a part.
RowsPlan rows_plan(const moqe_attention& at, const moqe_kv_batch& b, const moqe_kv_cache& c) {
  RowsPlan p;
  p.tiles = (static_cast<long long>(b.T) * (at.n_heads / c.n_heads) + rows_cols(c.head_dim) - 1) / rows_cols(c.head_dim);
  const long long sh = static_cast<long long>(b.S) * c.n_heads, tokens = static_cast<long long>(b.table_width) * c.block_tokens;
  const long long want = 512 / (sh * p.tiles), most = tokens / 1024;
  p.splits = static_cast<int>(want < most ? want : most);
  if (p.splits < 1) p.splits = 1;
  p.wgs = (sh + 7) / 8 * 8 * p.tiles * p.splits;
  return p;
}
}  // namespace

size_t kv_attend_rows_ws_bytes(const moqe_attention& at, const moqe_kv_batch& b, const moqe_kv_cache& c) {
  const RowsPlan p = rows_plan(at, b, c);
  if (p.splits == 1) return 0;
  const size_t rows = size_t(p.splits) * b.S * c.n_heads * (size_t(b.T) * (at.n_heads / c.n_heads));
  return align256(rows * 8) + align256(rows * c.head_dim * 4);
}

int32_t launch_kv_attend_rows(const void* q, long long q_stride, const moqe_attention& at, const moqe_kv_batch& b, const moqe_kv_cache& c,
                              void* out, long long out_stride, void* ws, hipStream_t st) {
  RowsArgs a{};
  a.q = static_cast<const uint16_t*>(q); a.out = static_cast<uint16_t*>(out); a.q_stride = q_stride; a.out_stride = out_stride;
  a.b = kv_batch_args(b);
  a.c = kv_cache_args(c);
  a.sc = KvScore{at.slopes, at.prefix, at.scale, at.cap, at.window};
  a.group = at.n_heads / c.n_heads;
  a.cols = b.T * a.group;
  const RowsPlan p = rows_plan(at, b, c);
  if (p.wgs >= (1ll << 31)) return set_error(MOQE_E_SHAPE, "moqe_kv_attention: %lld work-groups", p.wgs);
  a.tiles = int(p.tiles);
  a.splits = p.splits;
  if (p.splits > 1) a.parts = kv_parts(ws, size_t(p.splits) * b.S * c.n_heads * a.cols);
  const int lds = 64 * c.head_dim * 2 * 4;
  const dim3 grid(static_cast<unsigned>(p.wgs)), block(256);
  const bool extra = at.slopes || at.cap > 0.f || !(at.scale > 0.f);
  if (c.head_dim == 256) {
    const void* k = extra ? reinterpret_cast<const void*>(k_kv_attend_rows<256, true>) : reinterpret_cast<const void*>(k_kv_attend_rows<256, false>);
    const int32_t rc = ensure_dynamic_lds(extra ? LDSK_ATTEND_ROWS_EXTRA : LDSK_ATTEND_ROWS, k, lds, "moqe_kv_attention");
    if (rc) return rc;
  }
  ProfileScope ps(MOQE_PK_OTHER, st);
#define MOQE_ROWS(DH)                                                                         \
  do {                                                                                        \
    if (extra) hipLaunchKernelGGL((k_kv_attend_rows<DH, true>), grid, block, lds, st, a);     \
    else hipLaunchKernelGGL((k_kv_attend_rows<DH, false>), grid, block, lds, st, a);          \
  } while (0)
  if (c.head_dim == 64) MOQE_ROWS(64);
  else if (c.head_dim == 128) MOQE_ROWS(128);
  else MOQE_ROWS(256);
#undef MOQE_ROWS
  if (p.splits > 1) launch_kv_join(a.parts, a.b, a.c, c.head_dim, a.group, a.cols, p.splits, a.out, out_stride, st);
  return check_launch("kv_attention");
}

}  // namespace moqe
