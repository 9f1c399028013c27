// Block-sparse product with bias, activation and residual in its epilogue: the kernels of blast_bsr_spmm, whose sums go
// through an Epilogue (kern_common.h) on the way out, which costs the product what its operands' bytes cost: microseconds of the product
// alone / with bias / SiLU / bf16 residual / Z: 1600 x 6400 at 80 %, 64-wide, 333 tokens 10.6 / 10.5 / 11.1 / 11.2 / 11.2; 2048 x 8192
// at 90 %, 2048 tokens, fp32 15.6 / 15.6 / 15.7 / 16.2 / 16.6; 14336 x 4096 at 95 %, 128-wide, 4096 tokens, bf16 44.2 / 45.7 / 50.5 / 74.0
// / 61.5; one token, 6400 x 1600 3.5 whatever is asked for.  Bias and residual are loaded before the waves that share a tile meet
// (shared tiles, 333 tokens: 17.7 us when they were loaded after, 11.2).  Rows are never cut into chunks: the activation needs complete
// sums, and the result does not depend on the schedule.
#include "product_launch.h"

namespace {

// 32-bit offsets inside a tile's 256 rows, as y_fast.
bool rows_near(const void* p, int64_t ld) { return !p || (int64_t)257 * ld * 4 < ((int64_t)1 << 31); }
bool rows_together(int n, const void* p, int64_t ld, int64_t value_bytes) {
  return !p || (ld % n == 0 && blast::aligned(p, (size_t)(n * value_bytes)));
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
  e.pairs = rows_together(2, R, ldr, e.r_bf16 ? 2 : 4) && rows_together(2, Z, ldz, 2);
  e.quads = rows_together(4, R, ldr, e.r_bf16 ? 2 : 4) && rows_together(4, Z, ldz, 2);
  // feature-major operands, and pitches beyond 32-bit offsets, take the generic kernel
  if (layout != BLAST_TOKEN_MAJOR || !a.y_fast || !rows_near(R, ldr) || !rows_near(Z, ldz)) {
    switch (W->b) {
      case 16: return launch_tile<16, false>(a, stream, e);
      case 32: return launch_tile<32, false>(a, stream, e);
      case 64: return launch_tile<64, false>(a, stream, e);
      default: return launch_tile<128, false>(a, stream, e);
    }
  }
  if (group16_applies(W->b, layout, X, ldx, T) && ws && blast::aligned(ws, 16) && ws_bytes >= group16_bytes(W->cols, T)) {
    uint16_t* Xg = static_cast<uint16_t*>(ws);
    if (int rc = enqueue_group16(X, ldx, T, W->cols, Xg, stream)) return rc;
    a.X = Xg;
    a.x_grp16 = 1;
  }
  ChunkPlan plan{};  // (rows are never cut into chunks: the epilogue needs complete sums)
  plan.fullest = W->max_row_blocks;
  return dispatch_tile<false>(W->b, a, W->nnz, stream, plan, false, e);
}
