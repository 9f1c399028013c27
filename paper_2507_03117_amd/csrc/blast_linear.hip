// Block-sparse product with bias, activation and residual in its epilogue: the kernels of blast_bsr_spmm, whose sums go
// through an Epilogue (kern_common.h) on the way out.
#include "product_launch.h"

namespace {

template <int B>
int launch_linear_tile(TileArgs a, const Epilogue& e, hipStream_t stream) {
  using C = TileCfg<B>;
  a.ntt = (a.T + C::TT - 1) / C::TT;
  const int64_t grid = (int64_t)a.ntt * a.nbr;
  if (grid <= 0) return BLAST_OK;
  if (grid > INT32_MAX) return BLAST_ERR_INVALID_ARG;
  static blast::DeviceFlags lds_set;
  if (int rc = ensure_lds_limit(reinterpret_cast<const void*>(&k_linear_tile<B>), C::LDS_BYTES, lds_set)) return rc;
  k_linear_tile<B><<<dim3((unsigned)grid), dim3(256), C::LDS_BYTES, stream>>>(a, e);
  BLAST_LAUNCH_CHECK("k_linear_tile");
  return BLAST_OK;
}

}  // namespace

extern "C" int blast_bsr_linear(const blast_bsr_view* W, const uint16_t* X, int64_t ldx, int32_t layout, int64_t T,
                                const float* bias, int32_t act, const void* R, int64_t ldr, int32_t r_dtype, void* Y,
                                int64_t ldy, int32_t y_dtype, uint16_t* Z, int64_t ldz, void* ws, size_t ws_bytes,
                                void* stream_) {
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (int rc = check_view(W)) return rc;
  if (T < 0 || T > INT32_MAX / 2) return BLAST_ERR_INVALID_ARG;
  if (act < BLAST_ACT_NONE || act > BLAST_ACT_RELU) return BLAST_ERR_INVALID_ARG;
  if (y_dtype != BLAST_F32 && y_dtype != BLAST_BF16) return BLAST_ERR_INVALID_ARG;
  if (R && r_dtype != BLAST_F32 && r_dtype != BLAST_BF16) return BLAST_ERR_INVALID_ARG;
  if (int rc = check_dense(X, ldx, layout, W->cols, T)) return rc;
  if (int rc = check_dense(Y, ldy, layout, W->rows, T)) return rc;
  if (R)
    if (int rc = check_dense(R, ldr, layout, W->rows, T)) return rc;
  if (Z)
    if (int rc = check_dense(Z, ldz, layout, W->rows, T)) return rc;
  if (T == 0 || W->rows == 0) return BLAST_OK;
  TileArgs a{};
  a.m0 = mat_of(W);
  a.row_order = W->row_order;
  set_x(a, X, ldx, layout);
  set_y(a, Y, ldy, layout, y_dtype);
  a.T = (int)T;
  a.nbr = (int)(W->rows / W->b);
  a.kdim = W->cols;
  a.act = -1;  // (the epilogue has it)
  Epilogue e{};
  e.bias = bias;
  e.R = R;
  e.Z = Z;
  e.r_bf16 = r_dtype == BLAST_BF16;
  e.act = act;
  if (layout == BLAST_TOKEN_MAJOR) {
    e.srt = ldr, e.sri = 1, e.szt = ldz, e.szi = 1;
  } else {
    e.srt = 1, e.sri = ldr, e.szt = 1, e.szi = ldz;
  }
  (void)ws;
  (void)ws_bytes;
  switch (W->b) {
    case 16: return launch_linear_tile<16>(a, e, stream);
    case 32: return launch_linear_tile<32>(a, e, stream);
    case 64: return launch_linear_tile<64>(a, e, stream);
    default: return launch_linear_tile<128>(a, e, stream);
  }
}
