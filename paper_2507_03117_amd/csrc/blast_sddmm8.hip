// Gradient of the stored blocks from activations in scaled 8-bit form (kern_sddmm8.h).
#include "scaled8_check.h"

#include "kern_sddmm8.h"

using namespace blast_dev;

namespace {

// Forms and runs of tokens, from the sizes alone, so that the workspace does not depend on the device.
constexpr int64_t kCus = 256, kRunTokens = 512;

// 128-wide blocks by units where a workgroup to a block leaves CUs without one and four to a block give each wave enough, but not so many
// that what units read again counts (us, units first; 14336 x 4096 at 95 %, 179 blocks: 512 tokens 13.6 and 12.7, 1024: 19 and 24, 2048:
// 30 and 32, 4096: 54 and 49; 25 blocks, 2048 tokens: 11.4 and 15; 102 blocks, 8192 tokens: 62 and 56; 128, 4096: 39 and 35).
bool by_units(int32_t b, int64_t nnz, int64_t T) { return b == 64 || (nnz < 192 && T > 512 && nnz * T <= 192 * 2048); }

// A unit to a wave where there are many, or four waves to one (us, one wave first; 64-wide; 256 tokens, 768 units: 9.9 and 10.3, 1024:
// 10.4 and 11.5, 2048: 16 and 21; 2048 tokens, 1024 units: 42 and 40, 1536: 61 and 57, 2048: 64 and 74).
bool wave_each(int64_t units, int64_t T) { return units >= (T <= 512 ? 4 : 7) * kCus; }

int64_t token_runs(int32_t b, int64_t nnz, int64_t T) {
  const int64_t groups = by_units(b, nnz, T) ? nnz * (b / 64) * (b / 64) : nnz, fill = by_units(b, nnz, T) ? kCus : 2 * kCus;
  const int64_t want = groups > 0 ? fill / groups : 1, most = T / kRunTokens, runs = want < most ? want : most;
  return runs < 1 ? 1 : runs;
}

int check_structure(const blast_bsr_view* W, int64_t T) {
  if (!W || !W->row_ptr || W->rows < 0 || W->cols < 0 || W->nnz < 0 || W->nnz > INT32_MAX) return BLAST_ERR_INVALID_ARG;
  if (W->b != 64 && W->b != 128) return BLAST_ERR_UNSUPPORTED_BLOCK;
  if (W->rows % W->b || W->cols % W->b) return BLAST_ERR_SHAPE;
  if (W->rows > INT32_MAX / 2 || W->cols > INT32_MAX / 2 || T < 0 || T > INT32_MAX / 2) return BLAST_ERR_INVALID_ARG;
  return BLAST_OK;
}

template <int B, int FMT, int KW, int UPW>
int launch_units(const Sddmm8Args& a, hipStream_t stream) {
  using C = Sd8Units<B, KW, UPW>;
  static blast::DeviceFlags lds_set;
  int dev = 0;
  BLAST_HIP_TRY(hipGetDevice(&dev));
  if (!lds_set.test(dev)) {
    BLAST_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(&k_sddmm8_units<B, FMT, KW, UPW>),
                                      hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES));
    lds_set.set(dev);
  }
  const int64_t groups = ((int64_t)a.n_units + UPW - 1) / UPW;
  k_sddmm8_units<B, FMT, KW, UPW><<<dim3((unsigned)((groups + 7) / 8 * 8)), dim3(64 * C::NW), C::LDS_BYTES, stream>>>(a);
  BLAST_LAUNCH_CHECK("k_sddmm8_units");
  return BLAST_OK;
}

template <int FMT>
int launch(const Sddmm8Args& a, int32_t b, hipStream_t stream) {
  if (b == 64) return wave_each(a.n_units, a.T) ? launch_units<64, FMT, 1, 4>(a, stream) : launch_units<64, FMT, 4, 1>(a, stream);
  if (by_units(b, a.nnz, a.T)) return launch_units<128, FMT, 4, 1>(a, stream);
  k_sddmm8<FMT><<<dim3((unsigned)((int64_t)a.nnz * a.runs)), dim3(256), 0, stream>>>(a);
  BLAST_LAUNCH_CHECK("k_sddmm8");
  return BLAST_OK;
}

}  // namespace

extern "C" int blast_bsr_sddmm_scaled8_workspace(const blast_bsr_view* W, int64_t T, size_t* ws_bytes) {
  if (!ws_bytes) return BLAST_ERR_INVALID_ARG;
  if (int rc = check_structure(W, T)) return rc;
  const int64_t runs = token_runs(W->b, W->nnz, T);
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
  if (T == 0) {  // an empty sum
    const int64_t most = blast::most_groups(256) * 1024;  // values of a launch
    for (int64_t i = 0; i < n; i += most) {
      const int64_t part = n - i < most ? n - i : most;
      k_zero_blocks<<<dim3((unsigned)((part / 4 + 255) / 256)), dim3(256), 0, stream>>>(dvals + i, part);
    }
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
  int64_t runs = token_runs(W->b, W->nnz, T);
  a.run_tokens = (int)(((T + runs - 1) / runs + 63) / 64 * 64);
  runs = (T + a.run_tokens - 1) / a.run_tokens;
  const bool split = runs > 1;
  if (split && (!ws || !blast::aligned(ws, 16) || ws_bytes < (size_t)runs * (size_t)n * 4)) return BLAST_ERR_WORKSPACE;
  const int64_t units = W->nnz * (b / 64) * (b / 64) * runs;
  if (units > blast::most_groups(64)) return BLAST_ERR_INVALID_ARG;  // (a wave at least to each: more lanes than a launch has)
  a.runs = (int)runs;
  a.n_units = (int)units;
  a.out = split ? static_cast<float*>(ws) : dvals;
  a.out_run = n;
  if (int rc = a.x.fmt == BLAST_E4M3 ? launch<BLAST_E4M3>(a, b, stream) : launch<BLAST_E5M2>(a, b, stream)) return rc;
  if (!split) return BLAST_OK;
  k_join_runs<<<dim3((unsigned)((n / 4 + 255) / 256)), dim3(256), 0, stream>>>(a.out, n, a.runs, dvals, n);
  BLAST_LAUNCH_CHECK("k_join_runs");
  return BLAST_OK;
}
