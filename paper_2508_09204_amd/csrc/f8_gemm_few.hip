// Products of 8-bit rows and matrices, kernel for few rows: bound by reading the matrices once.
#include "f8_device.h"

namespace moqe {

// A work-group takes WT tiles of 16 features and MB blocks of 16 rows of an expert's bucket; its eight waves take every eighth block of 128 columns, straight from memory into operands (the
// next block's under way), and add their sums through LDS in a fixed order.
// One row, k 4096, onto 32000 features 23.4 us, 5.6 TB/s.  The tile kernel there 24.8; with more rows it wins (f8_shape()).
constexpr int FEW8_W = 8;
template <int MB, int WT, bool GATED, bool EXACT>
__global__ __launch_bounds__(FEW8_W * 64) void k_f8_few(F8Args a, uint32_t a_bytes, uint32_t as_bytes, uint32_t w_bytes) {
  constexpr int W = FEW8_W;
  __shared__ f8_f32x4 part[W][MB * WT][64];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, q = lane >> 4;
  const int e = blockIdx.y, t0 = blockIdx.x * WT, m0 = blockIdx.z * (MB * 16);
  const int2 bucket = f8_bucket(a, e);
  const int rows = bucket.y - m0;
  if (rows <= 0) return;
  const int blocks_m = min((rows + 15) / 16, MB);
  uint32_t x_at[MB], xs_at[MB];
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    const int src = max(f8_row(a, a.a_perm, bucket.x + m0 + min(m * 16 + r, rows - 1)), 0);
    x_at[m] = uint32_t(src) * a.a_stride + q * 16;
    xs_at[m] = uint32_t(src) * a.as_stride;
  }
  const auto a_rsrc = f8_rsrc(a.a, a_bytes), s_rsrc = f8_rsrc(a.a_scales, as_bytes), w_rsrc = f8_rsrc(a.w[e], w_bytes);
  uint32_t w_at[WT], ws_at[WT];
#pragma unroll
  for (int t = 0; t < WT; ++t) {
    const uint32_t nt = min(t0 + t, a.tiles - 1);
    w_at[t] = nt * uint32_t(a.blocks) * 2048;
    ws_at[t] = a.scale_off + nt * uint32_t(a.groups) * 64;
  }
  struct Block { F8Frag w[WT], x[MB]; uint32_t ws[WT], xs[MB]; };
  auto load = [&](Block& b, int kb) {
#pragma unroll
    for (int t = 0; t < WT; ++t) {
      b.w[t].u[0] = __builtin_bit_cast(f8_i32x4, __builtin_amdgcn_raw_buffer_load_b128(w_rsrc, lane * 16, int(w_at[t] + uint32_t(kb) * 2048), 0));
      b.w[t].u[1] = __builtin_bit_cast(f8_i32x4, __builtin_amdgcn_raw_buffer_load_b128(w_rsrc, lane * 16 + 1024, int(w_at[t] + uint32_t(kb) * 2048), 0));
      b.ws[t] = __builtin_amdgcn_raw_buffer_load_b8(w_rsrc, r * 4, int(ws_at[t] + uint32_t(kb >> 2) * 64 + (kb & 3)), 0);
    }
#pragma unroll
    for (int m = 0; m < MB; ++m)
      if (m < blocks_m) {
        b.x[m].u[0] = __builtin_bit_cast(f8_i32x4, __builtin_amdgcn_raw_buffer_load_b128(a_rsrc, int(x_at[m]), kb * 128, 0));
        b.x[m].u[1] = __builtin_bit_cast(f8_i32x4, __builtin_amdgcn_raw_buffer_load_b128(a_rsrc, int(x_at[m]) + 64, kb * 128, 0));
        b.xs[m] = __builtin_amdgcn_raw_buffer_load_b8(s_rsrc, int(xs_at[m]), kb, 0);
      }
  };
  f8_f32x4 acc[MB][WT];
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int t = 0; t < WT; ++t) acc[m][t] = f8_f32x4{0.f, 0.f, 0.f, 0.f};
  auto products = [&](const Block& b) {
    if constexpr (EXACT) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f8_bf16x8 we[WT];
#pragma unroll
        for (int t = 0; t < WT; ++t) we[t] = f8_quarter(b.w[t], i, f8_scale(b.ws[t]));
#pragma unroll
        for (int m = 0; m < MB; ++m)
          if (m < blocks_m) {
            const f8_bf16x8 xe = f8_quarter(b.x[m], i, f8_scale(b.xs[m]));
#pragma unroll
            for (int t = 0; t < WT; ++t) acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(we[t], xe, acc[m][t], 0, 0, 0);
          }
      }
    } else {
#pragma unroll
      for (int m = 0; m < MB; ++m)
        if (m < blocks_m) {
#pragma unroll
          for (int t = 0; t < WT; ++t) acc[m][t] = f8_mfma<0>(b.w[t], b.x[m], acc[m][t], b.ws[t], b.xs[m]);
        }
    }
  };
  Block b[2];
  if (wave < a.blocks) load(b[0], wave);
  for (int kb = wave; kb < a.blocks; kb += 2 * W) {
    if (kb + W < a.blocks) load(b[1], kb + W);
    products(b[0]);
    if (kb + W >= a.blocks) break;
    if (kb + 2 * W < a.blocks) load(b[0], kb + 2 * W);
    products(b[1]);
  }
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int t = 0; t < WT; ++t) part[wave][m * WT + t][lane] = acc[m][t];
  __syncthreads();
  constexpr int N = GATED ? 2 : 1, TASKS = MB * WT / N;
  for (int task = wave; task < TASKS; task += W) {
    const int m = task / (WT / N), t = task % (WT / N) * N, i = m * 16 + r;
    f8_f32x4 v[N];
#pragma unroll
    for (int c = 0; c < N; ++c) {
      v[c] = part[0][m * WT + t + c][lane];
#pragma unroll
      for (int w = 1; w < W; ++w) v[c] += part[w][m * WT + t + c][lane];
    }
    if constexpr (GATED) {
#pragma unroll
      for (int c = 0; c < 4; ++c) v[0][c] = f8_gated(v[0][c], v[N - 1][c]);
    }
    const int slot = bucket.x + m0 + i, n0 = (t0 + t) / N * 16 + q * 4;
    if (i >= rows || f8_row(a, a.a_perm, slot) < 0) continue;
    const int row = f8_row(a, a.y_perm, slot);
    if (row >= 0) f8_store(a, row, n0, v[0]);
  }
}

// fp32 rows in bucket order into 8-bit rows: 16 rows a work-group, a block of 128 features of each.  64 rows of 11008 5.6 us: a launch, since the tile kernel's work-groups hold fewer than 128
// features of a row there.
__global__ __launch_bounds__(256) void k_f8_quantize(F8Args a, const float* h) {
  const int lane = threadIdx.x & 15, slot = blockIdx.x * 16 + threadIdx.x / 16, f = blockIdx.y * F8_BLOCK + lane * 8;
  bool mine = false;
  for (int e = 0; e < a.K; ++e) {
    const int2 b = f8_bucket(a, e);
    mine = mine || (slot >= b.x && slot - b.x < b.y);
  }
  const int row = mine ? f8_row(a, a.y_perm, slot) : -1;
  if (row < 0 || f8_row(a, a.a_perm, slot) < 0) return;                   // all of the 16 lanes or none
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = f + i < a.n ? h[static_cast<long long>(slot) * a.n + f + i] : 0.f;
  const int e = f8_exponent(f8_row_top(f8_top(x)));
  *reinterpret_cast<uint2*>(a.y8 + row * a.y8_stride + f) = f8_codes(x, e);
  if (lane == 0) a.y8_scales[row * a.y8_scale_stride + blockIdx.y] = uint8_t(e + 127);
}

int32_t launch_f8_few(const F8Args& a, bool gated, bool exact, int blocks, int cols, hipStream_t st) {
  const long long M = static_cast<long long>(a.S) * a.T;
  const uint32_t a_bytes = uint32_t((M - 1) * a.a_stride + a.blocks * 128ll), as_bytes = uint32_t((M - 1) * a.as_stride + a.groups * 4ll);
  const uint32_t w_bytes = uint32_t(size_t(a.scale_off) + size_t(a.tiles) * a.groups * 64);
  auto go = [&](auto mbc, auto wtc) {
    constexpr int MB = decltype(mbc)::value, WT = decltype(wtc)::value;
    const dim3 grid((a.tiles + WT - 1) / WT, a.K, unsigned((M + MB * 16 - 1) / (MB * 16))), block(FEW8_W * 64);
    if constexpr (WT > 1) {
      if (gated && exact) hipLaunchKernelGGL((k_f8_few<MB, WT, true, true>), grid, block, 0, st, a, a_bytes, as_bytes, w_bytes);
      else if (gated) hipLaunchKernelGGL((k_f8_few<MB, WT, true, false>), grid, block, 0, st, a, a_bytes, as_bytes, w_bytes);
      if (gated) return;
    }
    if (exact) hipLaunchKernelGGL((k_f8_few<MB, WT, false, true>), grid, block, 0, st, a, a_bytes, as_bytes, w_bytes);
    else hipLaunchKernelGGL((k_f8_few<MB, WT, false, false>), grid, block, 0, st, a, a_bytes, as_bytes, w_bytes);
  };
  if (blocks == 2) go(std::integral_constant<int, 2>(), std::integral_constant<int, 2>());
  else if (cols == 2) go(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
  else go(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
  return check_launch("f8_gemm");
}

int32_t launch_f8_quantize(const F8Args& a, const float* h, hipStream_t st) {
  const long long M = static_cast<long long>(a.S) * a.T;
  hipLaunchKernelGGL(k_f8_quantize, dim3(unsigned((M + 15) / 16), f8_blocks(a.n)), dim3(256), 0, st, a, h);
  return check_launch("f8_gemm");
}

}  // namespace moqe
