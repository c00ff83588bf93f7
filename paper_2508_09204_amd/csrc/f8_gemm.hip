// Products of rows and matrices in 8-bit floating point: which kernel a call takes.
#include "dispatch_rules.h"
#include "f8_device.h"

namespace moqe {

size_t f8_gemm_ws_bytes(long long M, int n, int k, int K, bool gated, bool out8) {
  if (!out8 || M <= 0) return 0;
  const int tiles = f8_packed(n, k, gated).tiles;
  const bool needed = f8_through_workspace(f8_shape(M, K, tiles, gated, false)) || f8_through_workspace(f8_shape(M, K, tiles, gated, true));      // whatever sums a call takes
  return needed ? size_t(M) * n * 4 : 0;
}

int32_t launch_f8_gemm(const F8Args& a, bool gated, void* ws, hipStream_t st) {
  const F8Shape shape = f8_shape(static_cast<long long>(a.S) * a.T, a.K, a.tiles, gated, a.exact);
  const bool by_ws = a.y8 && f8_through_workspace(shape);
  F8Args p = a;
  if (by_ws) {                                            // fp32 rows in bucket order
    p.y8 = nullptr;
    p.y = ws; p.y_stride = a.n; p.y_bf16 = 0; p.y_perm = nullptr;
  }
  ProfileScope ps(MOQE_PK_OTHER, st);
  const int32_t rc = shape.rows == 0 ? launch_f8_few(p, gated, a.exact, shape.blocks, shape.cols, st) : launch_f8_tile(p, gated, a.exact, shape.rows, shape.cols, shape.parts, st);
  return rc || !by_ws ? rc : launch_f8_quantize(a, static_cast<const float*>(ws), st);
}

}  // namespace moqe
