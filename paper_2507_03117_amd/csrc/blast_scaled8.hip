// Activations and stored blocks into scaled 8-bit form and back (kern_scaled8.h).
#include "scaled8_check.h"

using namespace blast_dev;

namespace {

int check_keep(const void* X, int64_t ldx, int32_t dtype, int64_t T, int64_t K, const blast_scaled8_view* q) {
  if (T < 0 || T > INT32_MAX / 2 || K < 0 || K > INT32_MAX / 2) return BLAST_ERR_INVALID_ARG;
  if (dtype != BLAST_F32 && dtype != BLAST_BF16) return BLAST_ERR_INVALID_ARG;
  if (int rc = check_eight(q, T, K, 1)) return rc;
  if (T > 0 && K > 0 && (!X || ldx < K)) return BLAST_ERR_INVALID_ARG;
  return BLAST_OK;
}

int keep_args(const void* X, int64_t ldx, int32_t dtype, int64_t T, int64_t K, const blast_scaled8_view* q, KeepArgs& a, bool& vec, int64_t& grid) {
  a.q = eight_of(q);
  a.x = X;
  a.ldx = ldx;
  a.T = T;
  a.K = K;
  a.x_bf16 = dtype == BLAST_BF16;
  a.tiles = (int)((K + kKeepCols - 1) / kKeepCols);
  grid = a.tiles * ((T + 4 * kKeepRows - 1) / (4 * kKeepRows));
  vec = K % 8 == 0 && blast::aligned(X, 16) && ldx * (a.x_bf16 ? 2 : 4) % 16 == 0 && blast::aligned(q->codes, 8) && q->ld % 8 == 0;
  return grid > INT32_MAX ? BLAST_ERR_INVALID_ARG : BLAST_OK;
}

}  // namespace

extern "C" int blast_quantize_scaled8(const void* X, int64_t ldx, int32_t x_dtype, int64_t T, int64_t K, const blast_scaled8_view* out,
                                      void* stream_) {
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (int rc = check_keep(X, ldx, x_dtype, T, K, out)) return rc;
  if (T == 0 || K == 0) return BLAST_OK;
  KeepArgs a{};
  bool vec = false;
  int64_t grid = 0;
  if (int rc = keep_args(X, ldx, x_dtype, T, K, out, a, vec, grid)) return rc;
  const dim3 g((unsigned)grid), b(256);
  if (out->group == 64) {
    if (vec)
      k_quantize_scaled8<64, true><<<g, b, 0, stream>>>(a);
    else
      k_quantize_scaled8<64, false><<<g, b, 0, stream>>>(a);
  } else {
    if (vec)
      k_quantize_scaled8<128, true><<<g, b, 0, stream>>>(a);
    else
      k_quantize_scaled8<128, false><<<g, b, 0, stream>>>(a);
  }
  BLAST_LAUNCH_CHECK("k_quantize_scaled8");
  return BLAST_OK;
}

extern "C" int blast_dequantize_scaled8(const blast_scaled8_view* X, int64_t T, int64_t K, void* Y, int64_t ldy, int32_t y_dtype,
                                        void* stream_) {
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (int rc = check_keep(Y, ldy, y_dtype, T, K, X)) return rc;
  if (T == 0 || K == 0) return BLAST_OK;
  KeepArgs a{};
  bool vec = false;
  int64_t grid = 0;
  if (int rc = keep_args(Y, ldy, y_dtype, T, K, X, a, vec, grid)) return rc;
  if (vec)
    k_dequantize_scaled8<true><<<dim3((unsigned)grid), dim3(256), 0, stream>>>(a);
  else
    k_dequantize_scaled8<false><<<dim3((unsigned)grid), dim3(256), 0, stream>>>(a);
  BLAST_LAUNCH_CHECK("k_dequantize_scaled8");
  return BLAST_OK;
}

extern "C" int blast_bsr_quantize_scaled8(const blast_bsr_view* W, int32_t format, uint8_t* vals8, uint8_t* scales, void* stream_) {
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (!W || W->nnz < 0 || W->nnz > INT32_MAX || !format8_ok(format)) return BLAST_ERR_INVALID_ARG;
  if (W->b != 64 && W->b != 128) return BLAST_ERR_UNSUPPORTED_BLOCK;
  if (W->nnz == 0) return BLAST_OK;
  if (!W->vals || !blast::aligned(W->vals, 16) || !vals8 || !blast::aligned(vals8, 16) || !scales || !blast::aligned(scales, 16))
    return BLAST_ERR_INVALID_ARG;
  if (W->b == 64)
    k_quantize_blocks8<64><<<dim3((unsigned)W->nnz), dim3(256), 0, stream>>>(W->vals, W->nnz, format, vals8, scales);
  else
    k_quantize_blocks8<128><<<dim3((unsigned)W->nnz), dim3(256), 0, stream>>>(W->vals, W->nnz, format, vals8, scales);
  BLAST_LAUNCH_CHECK("k_quantize_blocks8");
  return BLAST_OK;
}
