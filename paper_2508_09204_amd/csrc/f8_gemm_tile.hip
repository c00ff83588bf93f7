// Products of 8-bit rows and matrices, tile kernel for many rows.
#include "f8_device.h"

namespace moqe {

typedef __attribute__((address_space(3))) void f8_lds;
__device__ __forceinline__ void f8_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
template <int VM> __device__ __forceinline__ void f8_wait() {          // at most VM memory requests and no LDS reads under way
  __builtin_amdgcn_s_waitcnt((VM & 15) | (7 << 4) | (0 << 8) | ((VM >> 4) << 14));
}

struct F8TileGeom {
  uint32_t a_bytes, as_bytes, w_bytes;       // sizes of the buffers, past which loads give zeros
  int32_t col_tiles;                         // work-groups along the features
  int32_t group;                             // row tiles that follow one another before the next column tile
};

// MB blocks of 16 rows, which all four waves share, by 4 NT tiles of 16 features, NT of each wave's own.  KS such groups of four waves share out the blocks of 128 columns.
// WD: blocks that a wave's weights are ahead.
template <int MB, int NT, int KS, int WD, int OUT, bool EXACT>
__global__ __launch_bounds__(256 * KS, KS == 1 ? 2 : 1) void k_f8_tile(F8Args a, F8TileGeom tg) {
  constexpr int ROWS = MB * 16, AL = (MB + 1) / 2, STAGED = ROWS < 32 ? 32 : ROWS;      // AL: requests of a wave for a block's activations
  constexpr int F = OUT == F8_PLAIN ? NT * 64 : NT * 32;                 // features of a work-group
  constexpr int BUF = STAGED * 128, SC = ROWS < 64 ? 64 : ROWS;
  __shared__ __attribute__((aligned(128))) uint8_t buf0_[KS * BUF], buf1_[KS * BUF], buf2_[KS * BUF], buf3_[KS * BUF];
  __shared__ uint32_t sc0_[KS * SC], sc1_[KS * SC];
  __shared__ int32_t dst[ROWS];
  const int part = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);      // of the columns
  const int tid = threadIdx.x & 255, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, q = lane >> 4;
  uint8_t *buf0 = buf0_ + part * BUF, *buf1 = buf1_ + part * BUF, *buf2 = buf2_ + part * BUF, *buf3 = buf3_ + part * BUF;
  uint32_t *sc0 = sc0_ + part * SC, *sc1 = sc1_ + part * SC;

  // which tile: the row tiles there are, dealt to the XCDs in runs, in groups of tg.group row tiles
  int rt = 0;
  for (int e = 0; e < a.K; ++e) rt += (f8_bucket(a, e).y + ROWS - 1) / ROWS;
  const int total = rt * tg.col_tiles, id = blockIdx.x;
  if (id >= total) return;
  const int each = total / 8, more = total - each * 8, xcd = id & 7, nth = id >> 3;
  const int at = xcd * each + min(xcd, more) + nth;
  if (nth >= each + (xcd < more ? 1 : 0)) return;
  const int per = tg.group * tg.col_tiles, gr = at / per, in = at - gr * per, rows_here = min(tg.group, rt - gr * tg.group);
  const int ct = in / rows_here;
  int tile = gr * tg.group + in - ct * rows_here, e = 0;
  int2 bucket = f8_bucket(a, 0);
  while (e + 1 < a.K) {
    const int tiles = (bucket.y + ROWS - 1) / ROWS;
    if (tile < tiles) break;
    tile -= tiles;
    bucket = f8_bucket(a, ++e);
  }
  const int m0 = tile * ROWS, m_left = bucket.y - m0;                   // rows of this tile

  // source and destination rows
  if (tid < ROWS) {
    const int m = bucket.x + m0 + tid;
    dst[tid] = tid < m_left && f8_row(a, a.a_perm, m) >= 0 ? f8_row(a, a.y_perm, m) : -1;
  }
  uint32_t a_at[AL];                                                     // of the rows that this lane stages: 8 rows a request, a lane's 16 bytes swizzled by its row
#pragma unroll
  for (int i = 0; i < AL; ++i) {
    const int row = (i * 4 + wave) * 8 + lane / 8;
    const int src = max(f8_row(a, a.a_perm, bucket.x + m0 + min(row, m_left - 1)), 0);
    a_at[i] = uint32_t(src) * a.a_stride + ((lane & 7) ^ (row & 7)) * 16;
  }
  const int sc_row = min(tid & (ROWS - 1), m_left - 1);
  const uint32_t sc_at = uint32_t(max(f8_row(a, a.a_perm, bucket.x + m0 + sc_row), 0)) * a.as_stride;
  const auto a_rsrc = f8_rsrc(a.a, tg.a_bytes), s_rsrc = f8_rsrc(a.a_scales, tg.as_bytes), w_rsrc = f8_rsrc(a.w[e], tg.w_bytes);
  const int blocks = a.blocks;
  uint32_t w_at[NT], ws_at[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const uint32_t nt = min(ct * (NT * 4) + wave * NT + t, a.tiles - 1);
    w_at[t] = nt * uint32_t(blocks) * 2048;
    ws_at[t] = a.scale_off + nt * uint32_t(a.groups) * 64;
  }

  auto stage = [&](uint8_t* buf, int kb) {
    const int k = min(kb, blocks - 1) * 128;
#pragma unroll
    for (int i = 0; i < AL; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(a_rsrc, (f8_lds*)(buf + (i * 4 + wave) * 1024), 16, int(a_at[i]), k, 0, 0);
  };
  auto stage_scales = [&](uint32_t* sc, int g) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(s_rsrc, (f8_lds*)(sc + (wave * 64 & (ROWS - 1))), 4, int(sc_at), min(g, a.groups - 1) * 4, 0, 0);
  };
  F8Frag w[WD + 1][NT];
  uint32_t ws[2][NT];
  auto load_w = [&](F8Frag (&f)[NT], int kb) {
    const uint32_t k = uint32_t(min(kb, blocks - 1)) * 2048;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f[t].u[0] = __builtin_bit_cast(f8_i32x4, __builtin_amdgcn_raw_buffer_load_b128(w_rsrc, lane * 16, int(w_at[t] + k), 0));
      f[t].u[1] = __builtin_bit_cast(f8_i32x4, __builtin_amdgcn_raw_buffer_load_b128(w_rsrc, lane * 16 + 1024, int(w_at[t] + k), 0));
    }
  };
  auto load_ws = [&](uint32_t (&s)[NT], int g) {
#pragma unroll
    for (int t = 0; t < NT; ++t) s[t] = uint32_t(__builtin_amdgcn_raw_buffer_load_b32(w_rsrc, r * 4, int(ws_at[t] + uint32_t(min(g, a.groups - 1)) * 64), 0));
  };

  f8_f32x4 acc[MB][NT];
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[m][t] = f8_f32x4{0.f, 0.f, 0.f, 0.f};

  const int each_g = (a.groups + KS - 1) / KS, g0 = part * each_g, kb0 = g0 * 4, steps = min(each_g * 4, blocks);       // of the first part, the longest
  stage_scales(sc0, g0);
  load_ws(ws[0], g0);
  stage(buf0, kb0);
  stage(buf1, kb0 + 1);
#pragma unroll
  for (int i = 0; i < WD; ++i) load_w(w[i], kb0 + i);

  // one block of 128 columns: products of step j of a group of four, the block after next on its way into LDS, the next one's weights into registers
  auto step = [&](auto jc, int kb, const uint8_t* cur, uint8_t* next2, const uint32_t* sc, const uint32_t (&wsc)[NT]) {
    constexpr int J = decltype(jc)::value, CUR = J & WD;
    stage(next2, kb + 2);
    load_w(w[(J + WD) & WD], kb + WD);
    if (KS > 1 && kb >= blocks) return;
    const uint8_t* p0 = cur + r * 128 + ((q ^ (r & 7)) * 16);
    const uint8_t* p1 = cur + r * 128 + (((q + 4) ^ (r & 7)) * 16);
    f8_bf16x8 we[EXACT ? NT : 1][4];
    if constexpr (EXACT) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) we[t][i] = f8_quarter(w[CUR][t], i, f8_scale(wsc[t] >> 8 * J));
    }
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      F8Frag x;
      x.u[0] = *reinterpret_cast<const f8_i32x4*>(p0 + m * 2048);
      x.u[1] = *reinterpret_cast<const f8_i32x4*>(p1 + m * 2048);
      const uint32_t xs = sc[m * 16 + r];
      if constexpr (EXACT) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f8_bf16x8 xe = f8_quarter(x, i, f8_scale(xs >> 8 * J));
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(we[t][i], xe, acc[m][t], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[m][t] = f8_mfma<J>(w[CUR][t], x, acc[m][t], wsc[t], xs);
      }
    }
  };
  auto sync = [&] {
    f8_wait<AL + (WD > 1 ? 4 : 2) * NT>();                               // the activations of two blocks ago have come; weights may be under way
    f8_barrier();
  };
  auto group = [&](int s, uint32_t* sc, uint32_t* sc_next, uint32_t (&wsc)[NT], uint32_t (&ws_next)[NT]) {
    const int kb = kb0 + s;
    sync();
    stage_scales(sc_next, (kb >> 2) + 1);
    load_ws(ws_next, (kb >> 2) + 1);
    step(std::integral_constant<int, 0>(), kb, buf0, buf2, sc, wsc);
    if (s + 1 >= steps) return;
    sync();
    step(std::integral_constant<int, 1>(), kb + 1, buf1, buf3, sc, wsc);
    if (s + 2 >= steps) return;
    sync();
    step(std::integral_constant<int, 2>(), kb + 2, buf2, buf0, sc, wsc);
    if (s + 3 >= steps) return;
    sync();
    step(std::integral_constant<int, 3>(), kb + 3, buf3, buf1, sc, wsc);
  };
  for (int s = 0; s < steps; s += 8) {
    group(s, sc0, sc1, ws[0], ws[1]);
    if (s + 4 < steps) group(s + 4, sc1, sc0, ws[1], ws[0]);
  }
  f8_wait<0>();
  f8_barrier();                                                          // nothing is on its way into LDS any more
  if constexpr (KS > 1) {                                                // the parts' sums, in their order
    static_assert((KS - 1) * NT <= 4 && KS >= 2, "a buffer for each part and tile");
    uint8_t* const bufs[4] = {buf0_, buf1_, buf2_, buf3_};
    auto at = [&](int p, int t) { return reinterpret_cast<f8_f32x4*>(bufs[(p - 1) * NT + t]) + wave * (MB * 64) + lane; };
#pragma unroll
    for (int p = 1; p < KS; ++p)
      if (part == p) {
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
          for (int t = 0; t < NT; ++t) at(p, t)[m * 64] = acc[m][t];
      }
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int p = 1; p < KS; ++p)
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[m][t] += at(p, t)[m * 64];
  }
  if constexpr (OUT != F8_GATED8) {
    constexpr int STEP = OUT == F8_PLAIN ? 1 : 2;
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      const int row = dst[m * 16 + r];
      if (row < 0) continue;
#pragma unroll
      for (int t = 0; t < NT; t += STEP) {
        f8_f32x4 v = acc[m][t];
        if constexpr (OUT == F8_GATED) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = f8_gated(acc[m][t][i], acc[m][t + STEP - 1][i]);
        }
        f8_store(a, row, ct * F + (wave * NT + t) / STEP * 16 + q * 4, v);
      }
    }
  } else {
    static_assert(NT == 4 && KS == 1, "a work-group's features are a block of 128");
    float* tops = reinterpret_cast<float*>(buf1);                        // [4][ROWS]
    f8_f32x4 h[MB][2];
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      float top = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = ct * F + (wave * 2 + t) * 16 + q * 4 + i < a.n ? f8_gated(acc[m][2 * t][i], acc[m][2 * t + 1][i]) : 0.f;
          h[m][t][i] = v;
          const float s = fabsf(v);
          top = s < INFINITY ? fmaxf(top, s) : top;
        }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (q == 0) tops[wave * ROWS + m * 16 + r] = top;
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      const int row = m * 16 + r;
      const float top = fmaxf(fmaxf(tops[row], tops[ROWS + row]), fmaxf(tops[2 * ROWS + row], tops[3 * ROWS + row]));
      const int ex = f8_exponent(top);
      const float both[8] = {h[m][0][0], h[m][0][1], h[m][0][2], h[m][0][3], h[m][1][0], h[m][1][1], h[m][1][2], h[m][1][3]};
      const uint2 c = f8_codes(both, ex);
      *reinterpret_cast<uint32_t*>(buf0 + row * 128 + wave * 32 + q * 4) = c.x;
      *reinterpret_cast<uint32_t*>(buf0 + row * 128 + wave * 32 + 16 + q * 4) = c.y;
      if (wave == 0 && q == 0 && dst[row] >= 0) a.y8_scales[dst[row] * a.y8_scale_stride + ct] = uint8_t(ex + 127);
    }
    __syncthreads();
    for (int u = tid; u < ROWS * 8; u += 256) {
      const int row = dst[u / 8];
      if (row >= 0) *reinterpret_cast<uint4*>(a.y8 + row * a.y8_stride + ct * 128 + (u & 7) * 16) = *reinterpret_cast<const uint4*>(buf0 + u * 16);
    }
  }
}

template <int MB, int NT, int KS, int WD, bool EXACT>
static int32_t launch_tile(const F8Args& a, bool gated, hipStream_t st) {
  const long long M = static_cast<long long>(a.S) * a.T;
  constexpr int ROWS = MB * 16;
  F8TileGeom tg{};
  tg.a_bytes = uint32_t((M - 1) * a.a_stride + a.blocks * 128ll);
  tg.as_bytes = uint32_t((M - 1) * a.as_stride + a.groups * 4ll);
  tg.w_bytes = uint32_t(size_t(a.scale_off) + size_t(a.tiles) * a.groups * 64);
  tg.col_tiles = (a.tiles + NT * 4 - 1) / (NT * 4);
  tg.group = 8;
  const long long rt = (M + ROWS - 1) / ROWS + a.K - 1, wgs = (rt * tg.col_tiles + 7) / 8 * 8;
  if (wgs >= (1ll << 23)) return set_error(MOQE_E_SHAPE, "moqe_f8_gemm: %lld work-groups", wgs);
  const dim3 grid(static_cast<unsigned>(wgs)), block(256 * KS);
  if (!gated) hipLaunchKernelGGL((k_f8_tile<MB, NT, KS, WD, F8_PLAIN, EXACT>), grid, block, 0, st, a, tg);
  else if (!a.y8) {
    if constexpr (NT > 1) hipLaunchKernelGGL((k_f8_tile<MB, NT, KS, WD, F8_GATED, EXACT>), grid, block, 0, st, a, tg);
  } else if constexpr (!EXACT && NT == 4) hipLaunchKernelGGL((k_f8_tile<MB, NT, KS, WD, F8_GATED8, false>), grid, block, 0, st, a, tg);
  return check_launch("f8_gemm");
}

// The tiles of f8_shape().  fp32 results: no 128 rows, whose operands in bf16 the registers do not hold.
int32_t launch_f8_tile(const F8Args& a, bool gated, bool exact, int rows, int cols, int parts, hipStream_t st) {
  if (exact) {
    if (cols == 16) return launch_tile<4, 4, 1, 1, true>(a, gated, st);
    if (cols == 8) return rows == 64 ? launch_tile<4, 2, 1, 3, true>(a, gated, st) : parts == 1 ? launch_tile<2, 2, 1, 3, true>(a, gated, st) : launch_tile<2, 2, 2, 3, true>(a, gated, st);
    return rows == 64 ? launch_tile<4, 1, 2, 3, true>(a, gated, st) : launch_tile<2, 1, 4, 3, true>(a, gated, st);
  }
  if (cols == 16) return rows == 128 ? launch_tile<8, 4, 1, 1, false>(a, gated, st) : launch_tile<4, 4, 1, 1, false>(a, gated, st);
  if (cols == 8) return rows == 64 ? launch_tile<4, 2, 1, 3, false>(a, gated, st) : parts == 1 ? launch_tile<2, 2, 1, 3, false>(a, gated, st) : launch_tile<2, 2, 2, 3, false>(a, gated, st);
  return rows == 64 ? launch_tile<4, 1, 2, 3, false>(a, gated, st) : launch_tile<2, 1, 4, 3, false>(a, gated, st);
}

}  // namespace moqe
