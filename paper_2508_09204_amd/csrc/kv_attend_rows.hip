// Attention over the 8-bit cache for many rows (prompts, chunks of prompts): bound by the matrix cores.
#include "kv_device.h"

namespace moqe {

struct RowsArgs {
  const uint16_t* q; uint16_t* out;
  long long q_stride, out_stride;
  KvBatch b; KvCache c; KvScore sc;
  int group, tiles;             // query heads to a key head; column tiles of a sequence and key head at most
};

// One work-group takes 128 columns (row i, query head g of the key head's group: column i * group + g), 32 for each of its four waves, through the
// tokens in tiles of 64.  The tile's codes become bf16 operands once, on their way into LDS (two buffers, one barrier a tile; the codes of the tile after
// next are already under way in registers), in the order in which a wave reads them: 16 bytes a lane in a row, no bank conflicts.  Scores stay in registers:
// the layout of S^T = K Q^T is the operand layout of O^T = V^T P^T.
template <int DH>
__global__ __launch_bounds__(256, 2) void k_kv_attend_rows(RowsArgs a) {
  constexpr int NC = 2, COLS = 128, KS = DH / 32, DT = DH / 16, U = DH / 64;   // U: 16-byte units of keys (and of values) a thread brings in
  constexpr int HALF = 64 * DH * 2;                                            // bytes of a tile's keys in bf16
  extern __shared__ __align__(16) uint8_t lds[];                               // [2][keys, values]
  __shared__ int nan_flag[2][4];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, r = lane & 15, kq = lane >> 4;
  // work-groups of one sequence and key head stay on one XCD (round robin over 8): its L2 holds their keys and values; the longest tiles go first
  const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  const int sh = slot / a.tiles * 8 + xcd;
  if (sh >= a.b.S * a.c.heads) return;
  const int h = sh % a.c.heads, s = sh / a.c.heads, tile = a.tiles - 1 - slot % a.tiles;
  const KvSeq q = kv_seq(a.b, s, a.c.bt_log2);
  const int rows = min(q.n, a.b.T), first_pos = q.first();
  const int i_first = tile * COLS / a.group;
  if (i_first >= rows) return;
  const int i_last = min((tile * COLS + COLS - 1) / a.group, rows - 1);
  const int prefix = a.sc.prefix ? min(a.sc.prefix[s], q.len) : 0, window = a.sc.window;
  const int seen = min(q.len, max(max(first_pos + i_last + 1, prefix), 0));
  const KvSteps ks = kv_steps(q.len, seen, first_pos + i_first, window, prefix);
  const float scale2 = a.sc.scale * KV_LOG2E;
  // the wave's own rows
  const int col0 = tile * COLS + wave * 32;
  const int w_first = first_pos + min(col0 / a.group, rows - 1), w_last = first_pos + min((col0 + 31) / a.group, rows - 1);
  const bool idle = col0 / a.group >= rows;

  kv_bf16x8 qf[NC][KS];
  int pos[NC];
  float slope[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int col = col0 + c * 16 + r, i = col / a.group, g = col - i * a.group;
    const bool in = i < rows;
    pos[c] = first_pos + i;
    slope[c] = in && a.sc.slopes ? a.sc.slopes[h * a.group + g] * KV_LOG2E : 0.f;
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
  const int tiles64 = (ks.count + 1) / 2;
  // lane i looks up step `look + i`
  int look = 0, ids = -1;
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
  // The tile under way: its codes, and of its two steps the scales, the first token (2^30: absent) and whether all rows of the work-group see all of it.
  uint4 kc[U], vc[U];
  float sk[2], sv[2];
  int t0n[2];
  auto fetch = [&](int t) {
    if (2 * t >= look + 64) { look += 64; look_up(); }
    int id[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      id[e] = __builtin_amdgcn_readlane(ids, (2 * t + e) & 63);
      sk[e] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scales), (2 * t + e) & 63));
      sv[e] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v_scales), (2 * t + e) & 63));
      t0n[e] = id[e] >= 0 ? ks.step(2 * t + e) * 32 : 1 << 30;
    }
#pragma unroll
    for (int n = 0; n < U; ++n) {
      const int u = n * 256 + tid, e = (n * 256 + (tid & ~63)) / (2 * DH);    // the step of this wave's units
      const int bid = __builtin_amdgcn_readfirstlane(e ? id[1] : id[0]);
      kc[n] = vc[n] = make_uint4(0, 0, 0, 0);
      if (bid >= 0) {
        const int tok = (e ? t0n[1] : t0n[0]) & ((1 << a.c.bt_log2) - 1);
        const long long at = (static_cast<long long>(bid) * a.c.heads + h) * block_bytes + tok * DH + (u % (2 * DH)) * 16;
        kc[n] = *reinterpret_cast<const uint4*>(a.c.k + at);
        vc[n] = *reinterpret_cast<const uint4*>(a.c.v + at);
      }
    }
  };
  auto put = [&](int buf) {
    uint8_t* kb = lds + buf * 2 * HALF;
    uint8_t* vb = kb + HALF;
    uint32_t any = 0;
#pragma unroll
    for (int n = 0; n < U; ++n) {
      const int u = n * 256 + tid, e = (n * 256 + (tid & ~63)) / (2 * DH);
      const float fk = e ? sk[1] : sk[0], fv = e ? sv[1] : sv[0];
      const int at = (u >> 6) * 2048 + lane * 16;           // a unit is two operands, 1 KB apart
      *reinterpret_cast<kv_bf16x8*>(kb + at) = kv_operand(kc[n].x, kc[n].y, fk);
      *reinterpret_cast<kv_bf16x8*>(kb + at + 1024) = kv_operand(kc[n].z, kc[n].w, fk);
      *reinterpret_cast<kv_bf16x8*>(vb + at) = kv_operand(vc[n].x, vc[n].y, fv);
      *reinterpret_cast<kv_bf16x8*>(vb + at + 1024) = kv_operand(vc[n].z, vc[n].w, fv);
#pragma unroll
      for (int y = 0; y < 4; ++y) any |= ((&vc[n].x)[y] & 0x7f7f7f7fu) + 0x01010101u;
    }
    const bool nan = __ballot((any & 0x80808080u) != 0) != 0;
    if (lane == 0) nan_flag[buf][wave] = nan;
  };

  int t0c[2];
  if (tiles64 > 0) {
    fetch(0);
    put(0);
    t0c[0] = t0n[0]; t0c[1] = t0n[1];
    if (tiles64 > 1) fetch(1);
  }
  __syncthreads();
  for (int t = 0; t < tiles64; ++t) {
    const int buf = t & 1;
    int t0[2] = {t0c[0], t0c[1]};
    if (t + 1 < tiles64) {
      put(buf ^ 1);
      t0c[0] = t0n[0]; t0c[1] = t0n[1];
      if (t + 2 < tiles64) fetch(t + 2);
    }
    bool any_seen = false, full = true;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      any_seen |= t0[e] < prefix || (t0[e] <= w_last && (window <= 0 || w_first - (t0[e] + 31) < window));
      full &= t0[e] + 31 < prefix || (t0[e] + 31 <= w_first && (window <= 0 || w_last - t0[e] < window));
    }
    if (!idle && any_seen) {
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
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            float v = sc[x][c][y];
            const int tok = t0[x / 2] + 16 * (x & 1) + 4 * kq + y;
            if (a.sc.cap > 0.f) v = kv_capped(v * a.sc.scale, a.sc.cap) * KV_LOG2E;
            else v *= scale2;
            if (a.sc.slopes) v -= slope[c] * fabsf(float(pos[c] - tok));
            if (!full && !kv_sees(tok, pos[c], q.len, prefix, window)) v = -INFINITY;
            sc[x][c][y] = v;
            top = fmaxf(top, v);
          }
        if (__any(top > m[c] + 8.f)) {       // the running maximum follows only where weights would pass 2^8: the sums are rescaled seldom
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float mn = fmaxf(m[c], top), f = exp2f(m[c] - mn);
          m[c] = mn;
          l[c] *= f;
#pragma unroll
          for (int d = 0; d < DT; ++d) o[c][d] *= f;
        }
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const float e = __builtin_amdgcn_exp2f(sc[x][c][y] - m[c]);
            l[c] += e;
            pf[c][x / 2][4 * (x & 1) + y] = static_cast<__bf16>(e);
          }
      }
      if (!full && (nan_flag[buf][0] | nan_flag[buf][1] | nan_flag[buf][2] | nan_flag[buf][3])) {
        // values that are NaN must not reach rows that do not see them (0 * NaN would): taken out of the product, counted over what a row sees
        for (int g = 0; g < 2; ++g) {
          kv_bf16x8 sees[NC];
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int y = 0; y < 8; ++y)
              sees[c][y] = static_cast<__bf16>(kv_sees((g ? t0[1] : t0[0]) + y / 4 * 16 + 4 * kq + y % 4, pos[c], q.len, prefix, window) ? 1.f : 0.f);
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            kv_bf16x8 vf = *reinterpret_cast<const kv_bf16x8*>(vb + (g * DT + d) * 1024), ones;
#pragma unroll
            for (int y = 0; y < 8; ++y) {
              const bool bad = !(float(vf[y]) == float(vf[y]));
              ones[y] = static_cast<__bf16>(bad ? 1.f : 0.f);
              vf[y] = bad ? static_cast<__bf16>(0.f) : vf[y];
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              o[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, g ? pf[c][1] : pf[c][0], o[c][d], 0, 0, 0);
              const kv_f32x4 cnt = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, sees[c], kv_f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
              for (int y = 0; y < 4; ++y) o[c][d][y] = cnt[y] > 0.f ? NAN : o[c][d][y];
            }
          }
        }
      } else {
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const kv_bf16x8 vf = *reinterpret_cast<const kv_bf16x8*>(vb + (g * DT + d) * 1024);
#pragma unroll
            for (int c = 0; c < NC; ++c) o[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[c][g], o[c][d], 0, 0, 0);
          }
      }
    }
    __syncthreads();
  }

#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] += __shfl_xor(l[c], 16);
    l[c] += __shfl_xor(l[c], 32);
    const float inv = l[c] == 0.f ? 0.f : 1.f / l[c];
    const int col = col0 + c * 16 + r, i = col / a.group, g = col - i * a.group;
    if (i < rows) {
      uint16_t* dst = a.out + (q.row0 + i) * a.out_stride + static_cast<long long>(h * a.group + g) * DH + kq * 4;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        uint32_t w[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const __bf16 u0 = static_cast<__bf16>(o[c][d][2 * y] * inv), u1 = static_cast<__bf16>(o[c][d][2 * y + 1] * inv);
          w[y] = uint32_t(__builtin_bit_cast(uint16_t, u0)) | uint32_t(__builtin_bit_cast(uint16_t, u1)) << 16;
        }
        *reinterpret_cast<uint2*>(dst + d * 16) = make_uint2(w[0], w[1]);
      }
    }
  }
}

int32_t launch_kv_attend_rows(const void* q, long long q_stride, const moqe_attention& at, const moqe_kv_batch& b, const moqe_kv_cache& c,
                              void* out, long long out_stride, hipStream_t st) {
  RowsArgs a{};
  a.q = static_cast<const uint16_t*>(q); a.out = static_cast<uint16_t*>(out); a.q_stride = q_stride; a.out_stride = out_stride;
  a.b = kv_batch_args(b);
  a.c = kv_cache_args(c);
  a.sc = KvScore{at.slopes, at.prefix, at.scale, at.cap, at.window};
  a.group = at.n_heads / c.n_heads;
  const long long tiles = (static_cast<long long>(b.T) * a.group + 127) / 128;
  const long long wgs = (static_cast<long long>(b.S) * c.n_heads + 7) / 8 * 8 * tiles;
  if (wgs >= (1ll << 31)) return set_error(MOQE_E_SHAPE, "moqe_kv_attention: %lld work-groups", wgs);
  a.tiles = int(tiles);
  const int lds = 64 * c.head_dim * 2 * 4;
  const dim3 grid(static_cast<unsigned>(wgs)), block(256);
  int32_t rc = MOQE_OK;
  if (c.head_dim == 256) rc = ensure_dynamic_lds(LDSK_ATTEND_ROWS, reinterpret_cast<const void*>(k_kv_attend_rows<256>), lds, "moqe_kv_attention");
  if (rc) return rc;
  ProfileScope ps(MOQE_PK_OTHER, st);
  if (c.head_dim == 64) hipLaunchKernelGGL((k_kv_attend_rows<64>), grid, block, lds, st, a);
  else if (c.head_dim == 128) hipLaunchKernelGGL((k_kv_attend_rows<128>), grid, block, lds, st, a);
  else hipLaunchKernelGGL((k_kv_attend_rows<256>), grid, block, lds, st, a);
  return check_launch("kv_attention");
}

}  // namespace moqe
