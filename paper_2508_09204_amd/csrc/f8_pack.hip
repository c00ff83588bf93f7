// Matrices in 8-bit floating point between rows and the order of the matrix cores' operands.
#include "f8_device.h"

namespace moqe {

struct F8PackArgs {
  uint8_t *codes[2], *scales[2];             // rows of w (and up)
  long long code_stride[2], scale_stride[2];
  uint8_t* packed;
  F8Packed p;
  int n, k, mats;
};

// A thread moves 16 codes, and of a tile's first 16 units' threads each a block's scale of its row.  Rows past n and columns past k are zeros in the packed matrix.
// Done once per matrix: bound by memory.  A matrix of 32000 x 4096 59 us.
template <bool PACK>
__global__ __launch_bounds__(256) void k_f8_pack(F8PackArgs a) {
  const unsigned long long unit = blockIdx.x * 256ull + threadIdx.x, tile = unit / 128;
  if (tile >= static_cast<unsigned long long>(a.p.tiles) * a.p.blocks) return;
  const int u = int(unit % 128), r = u % 16, col = u / 64 * 64 + u % 64 / 16 * 16;
  const int t = int(tile / a.p.blocks), b = int(tile % a.p.blocks), m = a.mats == 2 ? t & 1 : 0, row = (a.mats == 2 ? t >> 1 : t) * 16 + r;
  uint8_t* packed = a.packed + tile * 2048 + u * 16;
  uint8_t* scale = a.packed + f8_scale_at(a.p, t, r, b);
  if constexpr (PACK) {
    uint4 v = make_uint4(0, 0, 0, 0);
    uint8_t s = 7;                                   // 2^-120, as of a block of zeros
    if (row < a.n) {
      v = *reinterpret_cast<const uint4*>(a.codes[m] + row * a.code_stride[m] + b * F8_BLOCK + col);
      s = a.scales[m][row * a.scale_stride[m] + b];
      const int left = a.k - b * F8_BLOCK - col;     // columns of this unit
      uint32_t* w = &v.x;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] &= left >= 4 * i + 4 ? ~0u : left <= 4 * i ? 0u : (1u << 8 * (left - 4 * i)) - 1u;
    }
    *reinterpret_cast<uint4*>(packed) = v;
    if (u < 16) *scale = s;
  } else if (row < a.n) {
    *reinterpret_cast<uint4*>(a.codes[m] + row * a.code_stride[m] + b * F8_BLOCK + col) = *reinterpret_cast<const uint4*>(packed);
    if (u < 16) a.scales[m][row * a.scale_stride[m] + b] = *scale;
  }
}

namespace {
template <bool PACK>
int32_t launch(const moqe_f8_rows& w, const moqe_f8_rows* up, int n, int k, uint8_t* packed, hipStream_t st) {
  F8PackArgs a{};
  const moqe_f8_rows* rows[2] = {&w, up};
  a.mats = up ? 2 : 1;
  for (int m = 0; m < a.mats; ++m) {
    a.codes[m] = rows[m]->codes; a.scales[m] = rows[m]->scales;
    a.code_stride[m] = rows[m]->code_stride; a.scale_stride[m] = rows[m]->scale_stride;
  }
  a.packed = packed;
  a.p = f8_packed(n, k, up != nullptr);
  a.n = n; a.k = k;
  const unsigned long long wgs = (static_cast<unsigned long long>(a.p.tiles) * a.p.blocks + 1) / 2;      // below 2^20: a packed matrix has less than 4 GiB
  ProfileScope ps(MOQE_PK_OTHER, st);
  hipLaunchKernelGGL((k_f8_pack<PACK>), dim3(unsigned(wgs)), dim3(256), 0, st, a);
  return check_launch("f8_pack");
}
}  // namespace

int32_t launch_f8_pack(const moqe_f8_rows& w, const moqe_f8_rows* up, int n, int k, uint8_t* out, hipStream_t st) { return launch<true>(w, up, n, k, out, st); }
int32_t launch_f8_unpack(const moqe_f8_mat& m, const moqe_f8_rows& w, const moqe_f8_rows* up, hipStream_t st) {
  return launch<false>(w, up, m.n, m.k, const_cast<uint8_t*>(static_cast<const uint8_t*>(m.packed)), st);
}

}  // namespace moqe
