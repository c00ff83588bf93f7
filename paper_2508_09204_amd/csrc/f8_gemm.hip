// Products of rows and matrices in 8-bit floating point: which kernel a call takes.
#include "f8_device.h"

namespace moqe {

size_t f8_gemm_ws_bytes(long long M, int n, int, int, bool, bool out8) { return out8 ? size_t(M) * n * 4 : 0; }

int32_t launch_f8_gemm(const F8Args& a, bool gated, void* ws, hipStream_t st) {
  const long long M = static_cast<long long>(a.S) * a.T;
  const bool exact = !a.y8 && !a.y_bf16;                  // results that stay in fp32
  const bool few = M <= 64;
  const int shape = M >= 1024 ? 0 : 1;
  ProfileScope ps(MOQE_PK_OTHER, st);
  // rows in 8 bits need a block of 128 features in one work-group; where there is none, the result goes through the workspace
  const bool by_ws = a.y8 && (few || shape > 1);
  F8Args p = a;
  if (by_ws) {
    p.y8 = nullptr;
    p.y = ws; p.y_stride = a.n; p.y_bf16 = 0; p.wide = a.n % 4 == 0; p.y_perm = nullptr;
  }
  const int32_t rc = few ? launch_f8_few(p, gated, exact, M <= 16 ? 1 : M <= 32 ? 2 : 4, 2, st) : launch_f8_tile(p, gated, exact, shape, st);
  return rc || !by_ws ? rc : launch_f8_quantize(a, static_cast<const float*>(ws), st);
}

}  // namespace moqe
