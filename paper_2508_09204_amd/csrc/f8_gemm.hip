// Products of rows and matrices in 8-bit floating point: which kernel a call takes.
#include "dispatch_rules.h"
#include "f8_device.h"

namespace moqe {

size_t f8_gemm_ws_bytes(long long M, int n, int k, int K, bool gated, bool out8) {
  return out8 && M > 0 && f8_through_workspace(f8_shape(M, K, f8_packed(n, k, gated).tiles, gated, false)) ? size_t(M) * n * 4 : 0;
}

int32_t launch_f8_gemm(const F8Args& a, bool gated, void* ws, hipStream_t st) {
  const bool exact = !a.y8 && !a.y_bf16;                  // results that stay in fp32
  const F8Shape shape = f8_shape(static_cast<long long>(a.S) * a.T, a.K, a.tiles, gated, exact);
  const bool by_ws = a.y8 && f8_through_workspace(shape);
  F8Args p = a;
  if (by_ws) {                                            // fp32 rows in bucket order
    p.y8 = nullptr;
    p.y = ws; p.y_stride = a.n; p.y_bf16 = 0; p.y_perm = nullptr;
  }
  ProfileScope ps(MOQE_PK_OTHER, st);
  const int32_t rc = shape.rows == 0 ? launch_f8_few(p, gated, exact, shape.blocks, shape.cols, st) : launch_f8_tile(p, gated, exact, shape.rows, shape.cols, shape.parts, st);
  return rc || !by_ws ? rc : launch_f8_quantize(a, static_cast<const float*>(ws), st);
}

}  // namespace moqe
