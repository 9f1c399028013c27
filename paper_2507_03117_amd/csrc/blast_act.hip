// Gradient through an activation and a bias (kern_act.h).
#include "blast_common.h"

#include "kern_act.h"

using namespace blast_dev;

namespace {

bool pitch_ok(const void* p, int64_t ld, int64_t N) { return !p || ld >= N; }
bool pieces_ok(const void* p, int64_t ld, int64_t value_bytes) {
  return !p || (blast::aligned(p, 16) && ld * value_bytes % 16 == 0);
}

// Rows of a workgroup: from the sizes alone, so that the workspace does not depend on the device.
constexpr int64_t kWorkgroups = 2048;
int64_t run_rows(int64_t T, int64_t N) {
  const int64_t tiles = (N + kActCols - 1) / kActCols;
  const int64_t runs = (kWorkgroups + tiles - 1) / tiles;
  const int64_t rows = (T + runs - 1) / runs;
  return (rows + kActTeams - 1) / kActTeams * kActTeams;
}

// A workgroup owns its columns' sums up to this many rows, instead of a second launch that joins runs of rows: that launch and
// the gap before it take longer than the fewer workgroups lose.  GPU time alone from a graph, owned / joined, microseconds: GELU,
// 6400 columns, 64 rows 4.5 / 5.6, 333: 7.3 / 8.2, 512: 9.5 / 10.1, 1000: 13.5 / 13.3; two sums (more registers, fewer waves),
// 6400 columns, 64 rows 6.1 / 6.2, 128: 8.3 / 7.1; a call that waits for the launches saves another 3 to 5.  Not beyond 2^27 columns,
// whose owners (32 lanes to a column) would be 2^32 lanes: no launch has as many, and so many columns have their rows in one run.
bool columns_owned(int64_t T, int64_t N, int wanted) { return T <= (wanted > 1 ? 64 : 512) && N < ((int64_t)1 << 27) - 512; }

template <bool GATED, bool SUMS>
int launch(const ActArgs& a, bool vec, hipStream_t stream) {
  if constexpr (SUMS) {
    if (columns_owned(a.T, a.N, (a.sum_out[0] ? 1 : 0) + (a.sum_out[1] ? 1 : 0))) {
      const dim3 grid((unsigned)(((int64_t)a.N + 16 * kActOwned - 1) / (16 * kActOwned) * 16));
      // 256 threads hold 64 rows, two on their way: with 1024 three quarters have none (6400 columns, GELU, 256 / 1024 threads, 16
      // rows 4.0 / 4.8 us, 64: 4.5 / 5.2, 96: 5.4 / 5.2, 256: 8.5 / 6.2; 14336 columns, more workgroups than CUs, 64: 4.6 / 8.5, 128: 6.1 /
      // 8.8, 256: 10.1 / 11.8; two sums, 6400 columns, 64: 6.6 / 8.0)
      if (a.T <= 64) {
        if (vec)
          k_act_backward_columns<GATED, true, 256><<<grid, dim3(256), 0, stream>>>(a);
        else
          k_act_backward_columns<GATED, false, 256><<<grid, dim3(256), 0, stream>>>(a);
      } else {
        if (vec)
          k_act_backward_columns<GATED, true, 1024><<<grid, dim3(1024), 0, stream>>>(a);
        else
          k_act_backward_columns<GATED, false, 1024><<<grid, dim3(1024), 0, stream>>>(a);
      }
      BLAST_LAUNCH_CHECK("k_act_backward_columns");
      return BLAST_OK;
    }
  }
  const int64_t runs = (a.T + a.run - 1) / a.run, grid = runs * a.tiles;
  if (grid > INT32_MAX) return BLAST_ERR_INVALID_ARG;
  if (vec)
    k_act_backward<GATED, SUMS, true><<<dim3((unsigned)grid), dim3(256), 0, stream>>>(a);
  else
    k_act_backward<GATED, SUMS, false><<<dim3((unsigned)grid), dim3(256), 0, stream>>>(a);
  BLAST_LAUNCH_CHECK("k_act_backward");
  if (!SUMS || runs == 1) return BLAST_OK;
  JoinArgs j{};
  j.part = a.part;
  j.groups = (int)runs;
  j.width = a.N;
  int n = 0;
  for (int s = 0; s < 2; ++s)
    if (a.sum_out[s]) j.out[n++] = a.sum_out[s];
  k_join_sums<<<dim3((unsigned)((a.N + 63) / 64), (unsigned)n), dim3(1024), 0, stream>>>(j);
  BLAST_LAUNCH_CHECK("k_join_sums");
  return BLAST_OK;
}

}  // namespace

extern "C" int blast_act_backward_workspace(int64_t T, int64_t N, int32_t n_bias_grads, size_t* ws_bytes) {
  if (T < 0 || T > INT32_MAX / 2 || N < 0 || N > INT32_MAX / 2 || n_bias_grads < 0 || n_bias_grads > 2 || !ws_bytes)
    return BLAST_ERR_INVALID_ARG;
  *ws_bytes = 0;
  if (T == 0 || N == 0) return BLAST_OK;
  const int64_t rows = run_rows(T, N), runs = (T + rows - 1) / rows;
  if (runs > 1 && !columns_owned(T, N, n_bias_grads)) *ws_bytes = (size_t)n_bias_grads * (size_t)runs * (size_t)N * 4;
  return BLAST_OK;
}

extern "C" int blast_act_backward(const uint16_t* Z, int64_t ldz, const uint16_t* U, int64_t ldu, const void* dY,
                                  int64_t lddy, int32_t dy_dtype, int64_t T, int64_t N, int32_t act, uint16_t* dZ,
                                  int64_t lddz, uint16_t* dU, int64_t lddu, uint16_t* H, int64_t ldh, float* dbias_z,
                                  float* dbias_u, void* ws, size_t ws_bytes, void* stream_) {
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (T < 0 || T > INT32_MAX / 2 || N < 0 || N > INT32_MAX / 2) return BLAST_ERR_INVALID_ARG;
  if (act < BLAST_ACT_NONE || act > BLAST_ACT_RELU) return BLAST_ERR_INVALID_ARG;
  if (dy_dtype != BLAST_F32 && dy_dtype != BLAST_BF16) return BLAST_ERR_INVALID_ARG;
  const int wanted = (dbias_z ? 1 : 0) + (dbias_u ? 1 : 0);
  if (N == 0) return BLAST_OK;
  if (T == 0) {
    if (wanted == 0) return BLAST_OK;
    JoinArgs j{};
    j.width = (int)N;
    int n = 0;
    if (dbias_z) j.out[n++] = dbias_z;
    if (dbias_u) j.out[n++] = dbias_u;
    k_zero_sums<<<dim3((unsigned)((N + 255) / 256), (unsigned)n), dim3(256), 0, stream>>>(j);
    BLAST_LAUNCH_CHECK("k_zero_sums");
    return BLAST_OK;
  }
  const bool gated = U != nullptr;
  if (!dY || lddy < N) return BLAST_ERR_INVALID_ARG;
  if (!Z && (gated || act != BLAST_ACT_NONE)) return BLAST_ERR_INVALID_ARG;
  if (!gated && (dU || H || dbias_u)) return BLAST_ERR_INVALID_ARG;  // what does not exist has no gradient
  if (!pitch_ok(Z, ldz, N) || !pitch_ok(U, ldu, N) || !pitch_ok(dZ, lddz, N) || !pitch_ok(dU, lddu, N) || !pitch_ok(H, ldh, N))
    return BLAST_ERR_INVALID_ARG;
  size_t need = 0;
  if (int rc = blast_act_backward_workspace(T, N, wanted, &need)) return rc;
  if (need > 0 && (!ws || ws_bytes < need || !blast::aligned(ws, 16))) return BLAST_ERR_WORKSPACE;
  ActArgs a{};
  a.z = act == BLAST_ACT_NONE && !gated ? nullptr : Z;  // (not read)
  a.u = U;
  a.dy = dY;
  a.dz = dZ;
  a.du = dU;
  a.h = H;
  a.part = static_cast<float*>(ws);
  a.sum_out[0] = dbias_z;
  a.sum_out[1] = dbias_u;
  a.ldz = ldz;
  a.ldu = ldu;
  a.lddy = lddy;
  a.lddz = lddz;
  a.lddu = lddu;
  a.ldh = ldh;
  a.T = (int)T;
  a.N = (int)N;
  a.run = (int)run_rows(T, N);
  a.tiles = (int)((N + kActCols - 1) / kActCols);
  a.dy_bf16 = dy_dtype == BLAST_BF16;
  a.act = act;
  const bool vec = N % 8 == 0 && pieces_ok(a.z, ldz, 2) && pieces_ok(U, ldu, 2) && pieces_ok(dY, lddy, a.dy_bf16 ? 2 : 4) &&
                   pieces_ok(dZ, lddz, 2) && pieces_ok(dU, lddu, 2) && pieces_ok(H, ldh, 2);
  if (gated) return wanted ? launch<true, true>(a, vec, stream) : launch<true, false>(a, vec, stream);
  return wanted ? launch<false, true>(a, vec, stream) : launch<false, false>(a, vec, stream);
}
