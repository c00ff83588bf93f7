// Products of 8-bit rows and matrices, tile kernel for many rows.
#include "dispatch_rules.h"
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
//
// Activations go from memory to LDS directly, 16 bytes a lane swizzled by the row, so that operand reads are free of bank conflicts; weights never touch LDS, they lie in memory as the operands
// they are.  One barrier a block.  The scale of a row and block is the instruction's own operand, a byte of a dword that holds four blocks': nothing is multiplied.
// Fast sums are bound by the matrix cores, and by power: 8192 rows, k 11008, n 4096 in 270 to 290 us, 2560 to 2740 TFLOP/s at about 2 GHz (a library product in fp8 with one scale 2690 on 8192^3; nothing but products
// from registers 3900); the products take 60 % of the time that a SIMD has.  What it took:
//  * two work-groups to a CU (128 x 256, 251 registers) instead of one (256 x 256): 333 -> 299 us;
//  * memory requests spread over the row blocks' products: as one burst at the head of a block, products wait behind them in the wave's order of issue: 305 -> 286, 2048 rows of 4096 x 4096 41 -> 36;
//  * operands of the next row block read ahead of this one's products: 273 -> 270, 33.4 -> 31.4.
// No gain: activations three blocks ahead (7 % slower), priorities for products, groups of 16 row tiles, 32x32x64 products in a probe (no faster).
// EXACT: codes times scales as bf16 operands, 16x16x32 products: 4096^3 in 108 us, 1270 TFLOP/s, as a library bf16 product, 8192 rows, k 11008, n 4096 in 556, 1330; a wave converts its activations
// itself.
template <int MB, int NT, int KS, int WD, int OUT, bool EXACT>
__global__ __launch_bounds__(256 * KS, KS > 1 ? 1 : MB * NT <= 8 && !EXACT ? 3 : 2) void k_f8_tile(F8Args a, F8TileGeom tg) {
  constexpr int ROWS = MB * 16, AL = (MB + 1) / 2, STAGED = ROWS < 32 ? 32 : ROWS;      // AL: requests of a wave for a block's activations
  constexpr int F = OUT == F8_PLAIN ? NT * 64 : NT * 32;                 // features of a work-group
  constexpr int BUF = STAGED * 128;
  __shared__ __attribute__((aligned(128))) uint8_t buf0_[KS * BUF], buf1_[KS * BUF], buf2_[KS * BUF], buf3_[KS * BUF];
  __shared__ uint32_t scales_[KS][2][ROWS];                              // of a group of four blocks and the next
  __shared__ int32_t dst[ROWS];
  const int part = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);      // of the columns
  const int tid = threadIdx.x & 255, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, q = lane >> 4;
  uint8_t *buf0 = buf0_ + part * BUF, *buf1 = buf1_ + part * BUF, *buf2 = buf2_ + part * BUF, *buf3 = buf3_ + part * BUF;
  uint32_t (*scales)[ROWS] = scales_[part];

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

  auto stage_one = [&](uint8_t* buf, int kb, int i) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(a_rsrc, (f8_lds*)(buf + (i * 4 + wave) * 1024), 16, int(a_at[i]), min(kb, blocks - 1) * 128, 0, 0);
  };
  auto stage = [&](uint8_t* buf, int kb) {
#pragma unroll
    for (int i = 0; i < AL; ++i) stage_one(buf, kb, i);
  };
  uint32_t x_next = 0, ws[NT], ws_next[NT];                              // scales of the next group: of a row, of the features
  F8Frag w[WD + 1][NT];
  auto load_half = [&](F8Frag (&f)[NT], int kb, int i) {                   // half i & 1 of tile i / 2
    f[i / 2].u[i & 1] = __builtin_bit_cast(f8_i32x4, __builtin_amdgcn_raw_buffer_load_b128(w_rsrc, lane * 16 + (i & 1) * 1024, int(w_at[i / 2] + uint32_t(min(kb, blocks - 1)) * 2048), 0));
  };
  auto load_w = [&](F8Frag (&f)[NT], int kb) {
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) load_half(f, kb, i);
  };
  auto load_scales = [&](int g) {
    const int gg = min(g, a.groups - 1);
#pragma unroll
    for (int t = 0; t < NT; ++t) ws_next[t] = uint32_t(__builtin_amdgcn_raw_buffer_load_b32(w_rsrc, r * 4, int(ws_at[t] + uint32_t(gg) * 64), 0));
    x_next = uint32_t(__builtin_amdgcn_raw_buffer_load_b32(s_rsrc, int(sc_at), gg * 4, 0));
  };
  auto keep_scales = [&](int g) {
    if (ROWS >= 256 || tid < ROWS) scales[g & 1][tid & (ROWS - 1)] = x_next;
#pragma unroll
    for (int t = 0; t < NT; ++t) ws[t] = ws_next[t];
  };

  f8_f32x4 acc[MB][NT];
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[m][t] = f8_f32x4{0.f, 0.f, 0.f, 0.f};

  constexpr int AHEAD = 2, LOADS = AL + 2 * NT;
  const int each_g = (a.groups + KS - 1) / KS, g0 = part * each_g, kb0 = g0 * 4, steps = min(each_g * 4, blocks);       // of the first part, the longest
  load_scales(g0);
  stage(buf0, kb0);
  stage(buf1, kb0 + 1);
#pragma unroll
  for (int i = 0; i < WD; ++i) load_w(w[i], kb0 + i);
  keep_scales(g0);

  // A block of 128 columns: products of step J of a group of four, the block AHEAD on its way into LDS, the weights WD ahead into registers.
  auto step = [&](auto jc, int g) {
    constexpr int J = decltype(jc)::value, CUR = J & WD;
    const int kb = g * 4 + J;
    uint8_t* const bufs[4] = {buf0, buf1, buf2, buf3};
    // the activations of AHEAD blocks ago have come, and the scales stored in the step before; younger requests may be under way
    f8_wait<(AHEAD - 1) * AL + 2 * NT>();
    f8_barrier();
    if constexpr (J == 0) load_scales(g + 1);
    if constexpr (KS > 1) {
      load_w(w[(J + WD) & WD], kb + WD);
      stage(bufs[(J + AHEAD) & 3], kb + AHEAD);
      __builtin_amdgcn_sched_barrier(0);                                 // asked for before the products
    }
    if (kb < blocks) {                                                   // also what keeps a step in a block of its own: as one block of 128 products the registers do not hold them
      const uint32_t* sc = scales[g & 1];
      const uint8_t* p0 = bufs[J] + r * 128 + ((q ^ (r & 7)) * 16);
      const uint8_t* p1 = bufs[J] + r * 128 + (((q + 4) ^ (r & 7)) * 16);
      f8_bf16x8 we[EXACT ? NT : 1][4];
      if constexpr (EXACT) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) we[t][i] = f8_quarter(w[CUR][t], i, f8_scale(ws[t] >> 8 * J));
      }
      F8Frag x[2];
      uint32_t xs[2];
      auto read = [&](int m) {
        x[m & 1].u[0] = *reinterpret_cast<const f8_i32x4*>(p0 + m * 2048);
        x[m & 1].u[1] = *reinterpret_cast<const f8_i32x4*>(p1 + m * 2048);
        xs[m & 1] = sc[m * 16 + r];
      };
      read(0);
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        if (m + 1 < MB) read(m + 1);                                     // ahead of this one's products
        if constexpr (KS == 1) {                                         // a few requests ahead of each row block's products: all at once they keep the products waiting behind them
#pragma unroll
          for (int l = m * LOADS / MB; l < (m + 1) * LOADS / MB; ++l) {
            if (l < AL) stage_one(bufs[(J + AHEAD) & 3], kb + AHEAD, l);
            else load_half(w[(J + WD) & WD], kb + WD, l - AL);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (EXACT) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f8_bf16x8 xe = f8_quarter(x[m & 1], i, f8_scale(xs[m & 1] >> 8 * J));
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(we[t][i], xe, acc[m][t], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[m][t] = f8_mfma<J>(w[CUR][t], x[m & 1], acc[m][t], ws[t], xs[m & 1]);
        }
      }
    }
    if constexpr (J == 3) keep_scales(g + 1);
  };
  int g = g0;
  for (const int end = g0 + steps / 4; g < end; ++g) {
    step(std::integral_constant<int, 0>(), g);
    step(std::integral_constant<int, 1>(), g);
    step(std::integral_constant<int, 2>(), g);
    step(std::integral_constant<int, 3>(), g);
  }
  if (steps & 3) {
    step(std::integral_constant<int, 0>(), g);
    if ((steps & 3) > 1) step(std::integral_constant<int, 1>(), g);
    if ((steps & 3) > 2) step(std::integral_constant<int, 2>(), g);
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
  const dim3 grid(static_cast<unsigned>(f8_work_groups(F8Shape{ROWS, NT * 4, KS, 0}, M, a.K, a.tiles))), block(256 * KS);
  if (!gated) hipLaunchKernelGGL((k_f8_tile<MB, NT, KS, WD, F8_PLAIN, EXACT>), grid, block, 0, st, a, tg);
  else if (!a.y8) {
    if constexpr (NT > 1) hipLaunchKernelGGL((k_f8_tile<MB, NT, KS, WD, F8_GATED, EXACT>), grid, block, 0, st, a, tg);
  } else if constexpr (NT == 4) hipLaunchKernelGGL((k_f8_tile<MB, NT, KS, WD, F8_GATED8, EXACT>), grid, block, 0, st, a, tg);
  return check_launch("f8_gemm");
}

// The tiles of f8_shape().  Exact products: no 128 rows, whose operands in bf16 the registers do not hold.
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
