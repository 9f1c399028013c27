// Gradient of the stored blocks from activations in scaled 8-bit form (kern_sddmm8.h).
#include "scaled8_check.h"

#include "kern_sddmm8.h"

using namespace blast_dev;

namespace {

// Runs of tokens: from the sizes alone, so that the workspace does not depend on the device.
constexpr int64_t kWorkgroups = 512, kRunTokens = 512;
int64_t token_runs(int64_t nnz, int64_t T) {
  const int64_t want = nnz > 0 ? kWorkgroups / nnz : 1, most = T / kRunTokens;
  return want < most ? (want < 1 ? 1 : want) : (most < 1 ? 1 : most);
}

int check_structure(const blast_bsr_view* W, int64_t T) {
  if (!W || !W->row_ptr || W->rows < 0 || W->cols < 0 || W->nnz < 0 || W->nnz > INT32_MAX) return BLAST_ERR_INVALID_ARG;
  if (W->b != 64 && W->b != 128) return BLAST_ERR_UNSUPPORTED_BLOCK;
  if (W->rows % W->b || W->cols % W->b) return BLAST_ERR_SHAPE;
  if (W->rows > INT32_MAX / 2 || W->cols > INT32_MAX / 2 || T < 0 || T > INT32_MAX / 2) return BLAST_ERR_INVALID_ARG;
  return BLAST_OK;
}

}  // namespace

extern "C" int blast_bsr_sddmm_scaled8_workspace(const blast_bsr_view* W, int64_t T, size_t* ws_bytes) {
  if (!ws_bytes) return BLAST_ERR_INVALID_ARG;
  if (int rc = check_structure(W, T)) return rc;
  const int64_t runs = token_runs(W->nnz, T);
  *ws_bytes = runs > 1 ? (size_t)runs * (size_t)W->nnz * W->b * W->b * 4 : 0;
  return BLAST_OK;
}

extern "C" int blast_bsr_sddmm_scaled8(const blast_bsr_view* W, const uint16_t* dY, int64_t ldy, const blast_scaled8_view* X, int64_t T,
                                       float* dvals, void* ws, size_t ws_bytes, void* stream_) {
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (int rc = check_structure(W, T)) return rc;
  if (int rc = check_eight(X, T, W->cols, 16)) return rc;
  if (X->group < W->b) return BLAST_ERR_INVALID_ARG;
  if (W->nnz == 0) return BLAST_OK;
  if (!W->col_idx || !dvals || !blast::aligned(dvals, 16)) return BLAST_ERR_INVALID_ARG;
  const int b = W->b;
  const int64_t n = W->nnz * b * b;
  const dim3 each((unsigned)((n / 4 + 255) / 256));
  if (T == 0) {  // an empty sum
    k_zero_blocks<<<each, dim3(256), 0, stream>>>(dvals, n);
    BLAST_LAUNCH_CHECK("k_zero_blocks");
    return BLAST_OK;
  }
  if (W->rows == 0 || W->cols == 0) return BLAST_ERR_SHAPE;
  if (!dY || ldy < W->rows || ldy % 8 || !blast::aligned(dY, 16)) return BLAST_ERR_INVALID_ARG;
  Sddmm8Args a{};
  a.row_ptr = W->row_ptr;
  a.col_idx = W->col_idx;
  a.dy = dY;
  a.ldy = ldy;
  a.x = eight_of(X);
  a.T = (int)T;
  a.nbr = (int)(W->rows / b);
  a.nnz = (int)W->nnz;
  const int64_t stage = b == 128 ? Sd8Cfg<128>::TOK : Sd8Cfg<64>::TOK;
  int64_t runs = token_runs(W->nnz, T);
  a.run_tokens = (int)(((T + runs - 1) / runs + stage - 1) / stage * stage);
  runs = (T + a.run_tokens - 1) / a.run_tokens;
  const bool split = runs > 1;
  if (split && (!ws || !blast::aligned(ws, 16) || ws_bytes < (size_t)runs * (size_t)n * 4)) return BLAST_ERR_WORKSPACE;
  if (W->nnz * runs > INT32_MAX) return BLAST_ERR_INVALID_ARG;
  a.runs = (int)runs;
  a.out = split ? static_cast<float*>(ws) : dvals;
  a.out_run = n;
  const dim3 grid((unsigned)(W->nnz * runs));
  if (b == 64)
    k_sddmm8<64><<<grid, dim3(256), 0, stream>>>(a);
  else
    k_sddmm8<128><<<grid, dim3(256), 0, stream>>>(a);
  BLAST_LAUNCH_CHECK("k_sddmm8");
  if (!split) return BLAST_OK;
  k_join_runs<<<each, dim3(256), 0, stream>>>(a.out, n, a.runs, dvals, n);
  BLAST_LAUNCH_CHECK("k_join_runs");
  return BLAST_OK;
}
