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

int keep_args(const void* X, int64_t ldx, int32_t dtype, int64_t T, int64_t K, const blast_scaled8_view* q, KeepArgs& a, bool& vec) {
  a.q = eight_of(q);
  a.x = X;
  a.ldx = ldx;
  a.T = T;
  a.K = K;
  a.x_bf16 = dtype == BLAST_BF16;
  a.tiles = (int)((K + kKeepCols - 1) / kKeepCols);
  vec = K % 8 == 0 && blast::aligned(X, 16) && ldx * (a.x_bf16 ? 2 : 4) % 16 == 0 && blast::aligned(q->codes, 8) && q->ld % 8 == 0;
  return a.tiles * ((T + 4 * kKeepRows - 1) / (4 * kKeepRows)) > INT32_MAX ? BLAST_ERR_INVALID_ARG : BLAST_OK;
}

// f(arguments, grid) for as many tokens at a time as a launch has lanes for.
template <class F>
void for_tokens(KeepArgs a, F&& f) {
  constexpr int kRows = 4 * kKeepRows;
  const int64_t all = a.T, most = blast::most_groups(256) / a.tiles * kRows;
  for (int64_t t = 0; t < all; t += most) {
    a.T = all - t < most ? all - t : most;
    f(a, dim3((unsigned)(a.tiles * ((a.T + kRows - 1) / kRows))));
    a.q.codes += most * a.q.ld;
    a.q.scales += most;  // (a multiple of four: a wave's scales stay one word)
    a.x = static_cast<const unsigned char*>(a.x) + most * a.ldx * (a.x_bf16 ? 2 : 4);
  }
}

}  // namespace

extern "C" int blast_quantize_scaled8(const void* X, int64_t ldx, int32_t x_dtype, int64_t T, int64_t K, const blast_scaled8_view* out,
                                      void* stream_) {
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (int rc = check_keep(X, ldx, x_dtype, T, K, out)) return rc;
  if (T == 0 || K == 0) return BLAST_OK;
  KeepArgs args{};
  bool vec = false;
  if (int rc = keep_args(X, ldx, x_dtype, T, K, out, args, vec)) return rc;
  for_tokens(args, [&](const KeepArgs& a, dim3 g) {
    const dim3 b(256);
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
  });
  BLAST_LAUNCH_CHECK("k_quantize_scaled8");
  return BLAST_OK;
}

extern "C" int blast_dequantize_scaled8(const blast_scaled8_view* X, int64_t T, int64_t K, void* Y, int64_t ldy, int32_t y_dtype,
                                        void* stream_) {
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (int rc = check_keep(Y, ldy, y_dtype, T, K, X)) return rc;
  if (T == 0 || K == 0) return BLAST_OK;
  KeepArgs args{};
  bool vec = false;
  if (int rc = keep_args(Y, ldy, y_dtype, T, K, X, args, vec)) return rc;
  for_tokens(args, [&](const KeepArgs& a, dim3 g) {
    if (vec)
      k_dequantize_scaled8<true><<<g, dim3(256), 0, stream>>>(a);
    else
      k_dequantize_scaled8<false><<<g, dim3(256), 0, stream>>>(a);
  });
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
  const int64_t size = (int64_t)W->b * W->b, most = blast::most_groups(256);
  for (int64_t q = 0; q < W->nnz; q += most) {
    const int64_t n = W->nnz - q < most ? W->nnz - q : most;
    const dim3 g((unsigned)n), b(256);
    if (W->b == 64)
      k_quantize_blocks8<64><<<g, b, 0, stream>>>(W->vals + q * size, format, vals8 + q * size, scales + q);
    else
      k_quantize_blocks8<128><<<g, b, 0, stream>>>(W->vals + q * size, format, vals8 + q * size, scales + q);
  }
  BLAST_LAUNCH_CHECK("k_quantize_blocks8");
  return BLAST_OK;
}
