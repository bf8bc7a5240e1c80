// Root-mean-square norm with the residual's addition and 8-bit rows with
// scales, forward and backward.
#include "norm.hpp"

using namespace gg;

extern "C" int gg_rmsnorm_forward(const gg_rows_t* x, const gg_rows_t* res, int64_t n, int32_t dim,
                                  const void* w_d, int32_t w_dtype, float eps,
                                  const gg_rows_t* sum, const gg_rows_t* y, const gg_rows_t* q,
                                  float* rstd_d, hipStream_t stream) {
  NormArgs a = {};
  const int rc = pack_norm(x, res, n, dim, w_d, nullptr, w_dtype, eps, sum, y, q, nullptr, nullptr,
                           rstd_d, &a);
  if (rc != GG_OK || n == 0) return rc;
  return run_norm<false>(a, x->dtype, res, sum, stream);
}

extern "C" size_t gg_ws_rmsnorm(int64_t n, int32_t dim) {
  if (n < 0 || n > GG_NORM_MAX_ROWS || dim < 1 || dim > GG_NORM_MAX_DIM) return 0;
  return align_up((size_t)std::min<int64_t>(n, 1024) * dim * sizeof(float), 256);
}

extern "C" int gg_rmsnorm_backward(const gg_rows_t* dy, const gg_rows_t* dsum, const gg_rows_t* s,
                                   const float* rstd_d, int64_t n, int32_t dim, const void* w_d,
                                   int32_t w_dtype, const gg_rows_t* dx, float* dw_d, void* ws,
                                   size_t ws_bytes, hipStream_t stream) {
  return run_back<false>(dy, dsum, s, nullptr, rstd_d, n, dim, w_d, w_dtype, dx, dw_d, nullptr, ws,
                         ws_bytes, gg_ws_rmsnorm(n, dim), stream);
}
