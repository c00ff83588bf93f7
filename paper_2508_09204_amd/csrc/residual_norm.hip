// Norms before and after a block, fused with its gate and the residual: u = post(y), t = r + scale gate (.) u, r' = t, out = pre(t).
#include "f8_device.h"

#include <type_traits>

namespace moqe {

struct NormArgs {
  const void* y; const void* r; void* r_out; uint16_t* out; uint8_t *codes, *scales;
  const float *gate, *post_gain, *post_offset, *pre_gain, *pre_offset;
  long long ys, rs, ros, os, cs, ss;
  int M, d, gate_rows, post, pre, row_threads;
  float scale, post_eps, pre_eps;
};

__device__ __forceinline__ float bf16_up(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ __forceinline__ uint32_t bf16_round(float x) {
  const __bf16 b = static_cast<__bf16>(x);
  return uint32_t(__builtin_bit_cast(uint16_t, b));
}

// Eight values from feature f on, of a row or vector of d.  Rows that start anywhere (ODD: an odd d, stride or address) still take wide accesses, which need
// no alignment beyond an element's; only the last piece of an odd d goes element by element.
template <bool BF16> struct Values {
  uint4 q[BF16 ? 1 : 2];
  static constexpr int SIZE = BF16 ? 2 : 4;
};
template <bool BF16>
__device__ __forceinline__ void unpack(const Values<BF16>& w, float* v) {
  const uint32_t* u = &w.q[0].x;
  if constexpr (BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_up(u[i] & 0xffff); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float((i < 4 ? &w.q[0].x : &w.q[1].x)[i & 3]);
  }
}
template <bool BF16, bool ODD>
__device__ __forceinline__ void load_values(const void* base, long long at, int f, int d, float* v) {
  const char* p = static_cast<const char*>(base) + (at + f) * Values<BF16>::SIZE;
  if (!ODD || f + 8 <= d) {
    Values<BF16> w;
    if constexpr (ODD) __builtin_memcpy(&w, p, sizeof(w));
    else w = *reinterpret_cast<const Values<BF16>*>(p);
    unpack(w, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = 0.f;
      if (f + i < d) {
        if constexpr (BF16) v[i] = bf16_up(reinterpret_cast<const uint16_t*>(p)[i]);
        else v[i] = reinterpret_cast<const float*>(p)[i];
      }
    }
  }
}
template <bool BF16, bool ODD>
__device__ __forceinline__ void store_values(void* base, long long at, int f, int d, const float* v) {
  char* p = static_cast<char*>(base) + (at + f) * Values<BF16>::SIZE;
  if (!ODD || f + 8 <= d) {
    Values<BF16> w;
    if constexpr (BF16) {
      uint32_t u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = bf16_round(v[2 * i]) | bf16_round(v[2 * i + 1]) << 16;
      w.q[0] = make_uint4(u[0], u[1], u[2], u[3]);
    } else {
      w.q[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
      w.q[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    }
    if constexpr (ODD) __builtin_memcpy(p, &w, sizeof(w));
    else *reinterpret_cast<Values<BF16>*>(p) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (f + i < d) {
        if constexpr (BF16) reinterpret_cast<uint16_t*>(p)[i] = uint16_t(bf16_round(v[i]));
        else reinterpret_cast<float*>(p)[i] = v[i];
      }
  }
}

// Sum over the waves of a row, the same in all lanes: a butterfly in each wave, the waves' sums in their order.  `part`: a place of its own for each sum of a
// row, so that one barrier is enough.
__device__ __forceinline__ float row_sum(float v, int waves, float* part) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  if (waves > 1) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < waves; ++w) v += part[w];
  }
  return v;
}

// A row's values in the registers of its `th` threads: NV pieces of eight, piece j from feature (j * th + lane) * 8 on; zeros past the row's end.
template <int NV, bool ODD>
__device__ __forceinline__ void normed(float (&t)[NV][8], int d, int th, int lane, int kind, float eps, const float* gain, const float* offset, float* part) {
  float g[NV][8];                       // asked for before the sums are known, where registers allow it
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int f = (j * th + lane) * 8;
    if (NV <= 2 && gain && f < d) load_values<false, ODD>(gain, 0, f, d, g[j]);
  }
  float mean = 0.f;
  if (kind == MOQE_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) s += t[j][i];
    mean = row_sum(s, th / 64, part) / float(d);
  }
  float q = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int f = (j * th + lane) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      t[j][i] = f + (ODD ? i : 0) < d ? t[j][i] - mean : 0.f;
      q += t[j][i] * t[j][i];
    }
  }
  const float inv = 1.f / sqrtf(row_sum(q, th / 64, part + 16) / float(d) + eps);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int f = (j * th + lane) * 8;
    if (f < d) {
      float o[8];
      if (NV > 2 && gain) load_values<false, ODD>(gain, 0, f, d, g[j]);
      if (offset) load_values<false, ODD>(offset, 0, f, d, o);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        t[j][i] *= gain ? inv * g[j][i] : inv;
        if (offset) t[j][i] += o[i];
      }
    }
  }
}

// A row in the registers of a.row_threads threads, every input read once.  Rows of one wave need no barrier, and four share a work-group.
// F8: the result as 8-bit rows, besides bf16 ones if those are wanted too.  A block of 128 features is a piece of 16 neighbouring lanes.  64 rows of 4096 4.5 us (a launch); 32768 of 3584 with
// norms before and after 276, 4.7 TB/s: memory.  The arithmetic stays in fp32, as the sums are: all of it in 64 bits took 451 us there, for some codes of a million at the border of a rounding.
template <int NV, bool ODD, bool YBF, bool RBF, bool F8>
__global__ __launch_bounds__(1024) void k_residual_norm(NormArgs a) {
  __shared__ float part[4 * 16];
  const int th = a.row_threads, d = a.d, lane = th == 64 ? threadIdx.x & 63 : threadIdx.x;
  const uint32_t wg = blockIdx.y * gridDim.x + blockIdx.x, in_order = th == 64 ? wg * 4 + (threadIdx.x >> 6) : wg;
  if (in_order >= uint32_t(a.M)) return;
  const int row = static_cast<int>(in_order);
  float u[NV][8], t[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int f = (j * th + lane) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) u[j][i] = t[j][i] = 0.f;
    if (f < d) {
      if (a.y) load_values<YBF, ODD>(a.y, row * a.ys, f, d, u[j]);
      load_values<RBF, ODD>(a.r, row * a.rs, f, d, t[j]);
    }
  }
  if (a.y) {
    if (a.post != MOQE_NORM_NONE) normed<NV, ODD>(u, d, th, lane, a.post, a.post_eps, a.post_gain, a.post_offset, part);
    const float* gate = a.gate ? a.gate + (a.gate_rows > 0 ? static_cast<long long>(row / a.gate_rows) * d : 0) : nullptr;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int f = (j * th + lane) * 8;
      if (f < d) {
        float g[8];
        if (gate) load_values<false, ODD>(gate, 0, f, d, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[j][i] += a.scale * (gate ? g[i] * u[j][i] : u[j][i]);
      }
    }
  }
  if (a.r_out) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int f = (j * th + lane) * 8;
      if (f < d) store_values<RBF, ODD>(a.r_out, row * a.ros, f, d, t[j]);
    }
  }
  if (!F8 && !a.out) return;
  if (a.pre != MOQE_NORM_NONE) normed<NV, ODD>(t, d, th, lane, a.pre, a.pre_eps, a.pre_gain, a.pre_offset, part + 32);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int f = (j * th + lane) * 8;
    if ((!F8 || a.out) && f < d) store_values<true, ODD>(a.out, row * a.os, f, d, t[j]);
  }
  if constexpr (F8) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int f = (j * th + lane) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) t[j][i] = f + i < d ? t[j][i] : 0.f;
      const int e = f8_exponent(f8_row_top(f8_top(t[j])));
      if (f < f8_blocks(d) * F8_BLOCK) {
        *reinterpret_cast<uint2*>(a.codes + row * a.cs + f) = f8_codes(t[j], e);
        if ((threadIdx.x & 15) == 0) a.scales[row * a.ss + f / F8_BLOCK] = uint8_t(e + 127);
      }
    }
  }
}

namespace {
template <int NV, bool ODD>
void launch_types(const NormArgs& a, bool ybf, bool rbf, hipStream_t st) {
  const bool wave_rows = a.row_threads == 64;
  // a launch has fewer than 2^32 threads along x
  const uint32_t wgs = wave_rows ? (uint32_t(a.M) + 3) / 4 : uint32_t(a.M), gx = wgs < (1u << 20) ? wgs : 1u << 20;
  const dim3 grid(gx, (wgs + gx - 1) / gx), block(wave_rows ? 256 : a.row_threads);
  auto launch = [&](auto f8) {
    constexpr bool F8 = decltype(f8)::value;
    if (ybf && rbf) hipLaunchKernelGGL((k_residual_norm<NV, ODD, true, true, F8>), grid, block, 0, st, a);
    else if (ybf) hipLaunchKernelGGL((k_residual_norm<NV, ODD, true, false, F8>), grid, block, 0, st, a);
    else if (rbf) hipLaunchKernelGGL((k_residual_norm<NV, ODD, false, true, F8>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_residual_norm<NV, ODD, false, false, F8>), grid, block, 0, st, a);
  };
  if (a.codes) launch(std::true_type());
  else launch(std::false_type());
}
template <bool ODD>
void launch_pieces(NormArgs& a, bool ybf, bool rbf, hipStream_t st) {
  const int pieces = (a.d + 7) / 8;
  const int nv = pieces <= 1024 ? 1 : pieces <= 2048 ? 2 : 4;
  a.row_threads = ((pieces + nv - 1) / nv + 63) / 64 * 64;
  if (nv == 1) launch_types<1, ODD>(a, ybf, rbf, st);
  else if (nv == 2) launch_types<2, ODD>(a, ybf, rbf, st);
  else launch_types<4, ODD>(a, ybf, rbf, st);
}
}  // namespace

int32_t launch_residual_norm(const moqe_residual_step& s, const moqe_f8_rows* out8, hipStream_t st) {
  NormArgs a{};
  a.y = s.y; a.r = s.residual; a.r_out = s.residual_out; a.out = static_cast<uint16_t*>(s.out); a.gate = s.gate;
  a.post_gain = s.post.gain; a.post_offset = s.post.offset; a.pre_gain = s.pre.gain; a.pre_offset = s.pre.offset;
  a.ys = s.y_stride; a.rs = s.residual_stride; a.ros = s.residual_out_stride; a.os = s.out_stride;
  a.M = s.M; a.d = s.d; a.gate_rows = s.gate_rows; a.post = s.post.kind; a.pre = s.pre.kind;
  a.scale = s.scale; a.post_eps = s.post.eps; a.pre_eps = s.pre.eps;
  if (out8) { a.codes = out8->codes; a.scales = out8->scales; a.cs = out8->code_stride; a.ss = out8->scale_stride; }
  // 16-byte accesses where every row and vector starts on 16 bytes
  uintptr_t at = 0;
  for (const void* p : {s.y, s.residual, static_cast<const void*>(s.residual_out), static_cast<const void*>(s.out), static_cast<const void*>(s.gate),
                        static_cast<const void*>(s.post.gain), static_cast<const void*>(s.post.offset), static_cast<const void*>(s.pre.gain),
                        static_cast<const void*>(s.pre.offset)})
    at |= reinterpret_cast<uintptr_t>(p);
  int64_t strides = s.d | s.residual_stride;
  if (s.y) strides |= s.y_stride;
  if (s.residual_out) strides |= s.residual_out_stride;
  if (s.out) strides |= s.out_stride;
  ProfileScope ps(MOQE_PK_OTHER, st);
  const bool ybf = s.y_type == MOQE_TYPE_BF16, rbf = s.residual_type == MOQE_TYPE_BF16;
  if (at % 16 == 0 && strides % 8 == 0) launch_pieces<false>(a, ybf, rbf, st);
  else launch_pieces<true>(a, ybf, rbf, st);
  return check_launch("residual_norm");
}

}  // namespace moqe
