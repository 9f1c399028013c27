// Norms before and after a block with its gate and residual (kern_norm.h): entry points and the forward launches; those of the
// gradient are in norm_backward.h.
#include "blast_common.h"

#include "kern_norm.h"
#include "norm_backward.h"

using namespace blast_dev;

namespace {

bool dtype_ok(int32_t d) { return d == BLAST_F32 || d == BLAST_BF16; }
int64_t value_bytes(int32_t dtype) { return dtype == BLAST_BF16 ? 2 : 4; }

// An operand [T][width]: there, and with a pitch that holds a row.
bool rows_ok(const void* p, int64_t ld, int64_t width, int64_t T) { return T == 0 || (p && ld >= width); }

// 16- or 32-byte access to pieces of eight values.
bool pieces_ok(const void* p, int64_t ld, int32_t dtype) {
  return !p || (blast::aligned(p, 16) && ld * value_bytes(dtype) % 16 == 0);
}

int check_norm(const blast_norm_view* P, bool branch) {
  if (!P || P->width < 1 || P->width > BLAST_NORM_MAX_WIDTH) return BLAST_ERR_INVALID_ARG;
  if (P->kind != BLAST_NORM_RMS && P->kind != BLAST_NORM_LAYER) return BLAST_ERR_INVALID_ARG;
  if (P->post != 0 && P->post != 1) return BLAST_ERR_INVALID_ARG;
  if (P->kind == BLAST_NORM_RMS && (P->bias || (P->post && P->post_bias))) return BLAST_ERR_INVALID_ARG;
  if (!(P->eps >= 0.0f) || !dtype_ok(P->p_dtype) || !dtype_ok(P->g_dtype)) return BLAST_ERR_INVALID_ARG;
  if (branch && P->gate && P->ldg != 0 && P->ldg < P->width) return BLAST_ERR_INVALID_ARG;
  return BLAST_OK;
}

// What the view says, with the branch's part left out where there is none.
NormArgs args_of(const blast_norm_view* P, bool branch, int64_t T) {
  NormArgs a{};
  a.T = T;
  a.width = (int)P->width;
  a.layer = P->kind == BLAST_NORM_LAYER;
  a.post = branch ? P->post : 0;
  a.eps = P->eps;
  a.scale = P->scale;
  a.p_bf16 = P->p_dtype == BLAST_BF16;
  a.g_bf16 = P->g_dtype == BLAST_BF16;
  a.w = P->weight;
  a.b = P->bias;
  if (a.post) {
    a.pw = P->post_weight;
    a.pb = P->post_bias;
  }
  if (branch) {
    a.gate = P->gate;
    a.ldg = P->ldg;
  }
  return a;
}

bool params_pieces_ok(const NormArgs& a) {
  return a.width % 8 == 0 && blast::aligned(a.w, 16) && blast::aligned(a.b, 16) && blast::aligned(a.pw, 16) &&
         blast::aligned(a.pb, 16) && pieces_ok(a.gate, a.ldg, a.g_bf16 ? BLAST_BF16 : BLAST_F32);
}

const void* row_at(const void* p, int64_t at, int bf16) { return static_cast<const char*>(p) + at * (bf16 ? 2 : 4); }
void* row_at(void* p, int64_t at, int bf16) { return static_cast<char*>(p) + at * (bf16 ? 2 : 4); }

// The call without its first n rows.
NormArgs rows_after(NormArgs a, int64_t n) {
  a.T -= n;
  a.h = row_at(a.h, n * a.ldh, a.h_bf16);
  a.x = row_at(a.x, n * a.ldx, a.x_bf16);
  if (a.y) {
    a.y = row_at(a.y, n * a.ldy, a.y_bf16);
    a.h_out = row_at(a.h_out, n * a.ldho, a.h_bf16);
    if (a.gate) a.gate = row_at(a.gate, n * a.ldg, a.g_bf16);
  }
  if (a.stats) a.stats += n * 4;
  return a;
}

// A row (with one wave to a row, four) to a workgroup while several workgroups fit on a CU: the others' loads cover one's
// sums (16 waves a CU that go over the rows, one ahead / a row each, microseconds: 4096 x 4096, branch with a norm 29.8 / 26.0; 2048
// x 8192 33.3 / 31.1; one row of 4096 3.5 / 3.0).  Rows of more than 8192 take a CU for themselves: a workgroup per CU goes over them, one
// ahead (2048 x 16384, gate per token 80.1 / 66.0; layer norms 85.9 / 67.3).
template <int NW, int NCH, bool VEC, bool AHEAD = false, bool LOW = false>
int launch_forward(const NormArgs& a, hipStream_t stream) {
  constexpr int kRows = NW == 1 ? 4 : 1;
  constexpr int kThreads = NW == 1 ? 256 : 64 * NW;
  constexpr int64_t kMostRows = ((int64_t)1 << 31) / kThreads * kRows;  // of a launch (fewer than 2^32 lanes)
  if (NW * NCH <= 16 && a.T > kMostRows) {
    NormArgs part = a;
    part.T = kMostRows;
    if (int rc = launch_forward<NW, NCH, VEC, AHEAD, LOW>(part, stream)) return rc;
    return launch_forward<NW, NCH, VEC, AHEAD, LOW>(rows_after(a, kMostRows), stream);
  }
  const int64_t grid = (a.T + kRows - 1) / kRows;
  if (NW * NCH > 16 && grid > 256) {
    k_norm_residual<NW, NCH, VEC, (NW * NCH > 16), AHEAD, LOW><<<dim3(256), dim3(kThreads), 0, stream>>>(a);
  } else {
    k_norm_residual<NW, NCH, VEC, false, false, LOW><<<dim3((unsigned)grid), dim3(kThreads), 0, stream>>>(a);
  }
  BLAST_LAUNCH_CHECK("k_norm_residual");
  return BLAST_OK;
}

int dispatch_forward(const NormArgs& a, bool vec, hipStream_t stream) {
  if (!vec) {
    if (a.width <= 2048) return launch_forward<4, 1, false>(a, stream);
    return a.width <= 8192 ? launch_forward<16, 1, false>(a, stream) : launch_forward<16, 4, false>(a, stream);
  }
  if (a.width <= 512) return launch_forward<1, 1, true>(a, stream);
  if (a.width <= 1024) return launch_forward<2, 1, true>(a, stream);
  if (a.width <= 2048) return launch_forward<4, 1, true>(a, stream);
  if (a.width <= 4096) return launch_forward<8, 1, true>(a, stream);
  if (a.width <= 8192) return launch_forward<16, 1, true>(a, stream);
  // (every operand that the kernel converts: a weight or a bias may be there without the other, and pw, pb are null without a branch)
  const bool low = a.h_bf16 && ((!a.w && !a.b && !a.pw && !a.pb) || a.p_bf16) && (!a.y || (a.y_bf16 && (!a.gate || a.g_bf16)));
  if (a.width <= 16384) return low ? launch_forward<16, 2, true, true, true>(a, stream) : launch_forward<16, 2, true>(a, stream);
  return launch_forward<16, 4, true>(a, stream);
}

}  // namespace

extern "C" int blast_norm_residual(const blast_norm_view* P, const void* h, int64_t ldh, int32_t h_dtype, const void* y,
                                   int64_t ldy, int32_t y_dtype, int64_t T, void* h_out, int64_t ldho, void* x, int64_t ldx,
                                   int32_t x_dtype, float* stats, void* stream_) {
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  const bool branch = y != nullptr;
  if (int rc = check_norm(P, branch)) return rc;
  if (T < 0 || T > INT32_MAX / 2) return BLAST_ERR_INVALID_ARG;
  if (!dtype_ok(h_dtype) || !dtype_ok(x_dtype) || (branch && !dtype_ok(y_dtype))) return BLAST_ERR_INVALID_ARG;
  if (T == 0) return BLAST_OK;
  const int64_t E = P->width;
  if (!rows_ok(h, ldh, E, T) || !rows_ok(x, ldx, E, T)) return BLAST_ERR_INVALID_ARG;
  if (branch && (!rows_ok(y, ldy, E, T) || !rows_ok(h_out, ldho, E, T))) return BLAST_ERR_INVALID_ARG;
  if (stats && !blast::aligned(stats, 16)) return BLAST_ERR_INVALID_ARG;
  NormArgs a = args_of(P, branch, T);
  a.h = h;
  a.ldh = ldh;
  a.h_bf16 = h_dtype == BLAST_BF16;
  a.x = x;
  a.ldx = ldx;
  a.x_bf16 = x_dtype == BLAST_BF16;
  a.stats = stats;
  bool vec = params_pieces_ok(a) && pieces_ok(h, ldh, h_dtype) && pieces_ok(x, ldx, x_dtype);
  if (branch) {
    a.y = y;
    a.ldy = ldy;
    a.y_bf16 = y_dtype == BLAST_BF16;
    a.h_out = h_out;
    a.ldho = ldho;
    a.past = T * P->width * (a.h_bf16 ? 2 : 4) >= kPastBytes;
    vec = vec && pieces_ok(y, ldy, y_dtype) && pieces_ok(h_out, ldho, h_dtype);
  }
  return dispatch_forward(a, vec, stream);
}

extern "C" int blast_norm_residual_backward_workspace(const blast_norm_view* P, int64_t T, size_t* ws_bytes) {
  if (int rc = check_norm(P, true)) return rc;
  if (T < 0 || T > INT32_MAX / 2 || !ws_bytes) return BLAST_ERR_INVALID_ARG;
  const int layer = P->kind == BLAST_NORM_LAYER;
  const int sums = 1 + layer + (P->post ? 1 + layer : 0) + (P->gate && P->ldg == 0 ? 1 : 0);
  // (without a branch fewer sums are wanted: the size serves that call as well)
  const int64_t groups = T <= blast::kBackwardRows ? T : blast::kBackwardGroups;
  const bool owned = T <= 1 || blast::columns_owned(T, true, P->post, P->gate && P->ldg == 0);
  *ws_bytes = owned ? 0 : (size_t)sums * (size_t)groups * (size_t)P->width * 4;
  return BLAST_OK;
}

extern "C" int blast_norm_residual_backward(const blast_norm_view* P, const void* h_out, int64_t ldho, int32_t h_dtype,
                                            const void* y, int64_t ldy, int32_t y_dtype, const float* stats, const void* dx,
                                            int64_t lddx, int32_t dx_dtype, const void* dh_out, int64_t lddho, int64_t T,
                                            void* dh, int64_t lddh, void* dy, int64_t lddy, int32_t dy_dtype, void* dgate,
                                            int64_t lddg, float* dweight, float* dbias, float* dpost_weight,
                                            float* dpost_bias, void* ws, size_t ws_bytes, void* stream_) {
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  // (over no rows the operands may be null, so the branch then goes by what is asked for)
  const bool branch = y != nullptr || (T == 0 && (dy || dgate || dpost_weight || dpost_bias));
  if (int rc = check_norm(P, branch)) return rc;
  if (T < 0 || T > INT32_MAX / 2) return BLAST_ERR_INVALID_ARG;
  if (!dtype_ok(h_dtype) || !dtype_ok(dx_dtype)) return BLAST_ERR_INVALID_ARG;
  if ((branch && T > 0 && !dtype_ok(y_dtype)) || (dy && !dtype_ok(dy_dtype))) return BLAST_ERR_INVALID_ARG;
  const int64_t E = P->width;
  // what does not exist has no gradient; the weight and bias have one with or without a branch
  if (!branch && (dy || dgate || dpost_weight || dpost_bias)) return BLAST_ERR_INVALID_ARG;
  if (dgate && !P->gate) return BLAST_ERR_INVALID_ARG;
  if ((dpost_weight || dpost_bias) && !P->post) return BLAST_ERR_INVALID_ARG;
  if ((dbias || dpost_bias) && P->kind != BLAST_NORM_LAYER) return BLAST_ERR_INVALID_ARG;
  NormArgs a = args_of(P, branch, T);
  const bool gate_sum = dgate && P->ldg == 0;
  a.sum_out[0] = dweight;
  a.sum_out[1] = dbias;
  a.sum_out[2] = gate_sum ? static_cast<float*>(dgate) : nullptr;
  a.sum_out[3] = dpost_weight;
  a.sum_out[4] = dpost_bias;
  if (T == 0) {
    JoinArgs j{};
    j.width = (int)E;
    int n = 0;
    for (int s = 0; s < kNormSums; ++s)
      if (a.sum_out[s]) j.out[n++] = a.sum_out[s];
    if (n == 0) return BLAST_OK;
    k_zero_sums<<<dim3((unsigned)((E + 255) / 256), (unsigned)n), dim3(256), 0, stream>>>(j);
    BLAST_LAUNCH_CHECK("k_zero_sums");
    return BLAST_OK;
  }
  if (!rows_ok(h_out, ldho, E, T) || !rows_ok(dx, lddx, E, T) || !rows_ok(dh, lddh, E, T)) return BLAST_ERR_INVALID_ARG;
  if (branch && !rows_ok(y, ldy, E, T)) return BLAST_ERR_INVALID_ARG;
  if ((dh_out && lddho < E) || (dy && lddy < E) || (dgate && !gate_sum && lddg < E)) return BLAST_ERR_INVALID_ARG;
  if (!stats || !blast::aligned(stats, 16)) return BLAST_ERR_INVALID_ARG;
  size_t need = 0;
  if (int rc = blast_norm_residual_backward_workspace(P, T, &need)) return rc;
  if (!branch && blast::columns_owned(T, false, 0, false)) need = 0;
  if (need > 0 && (!ws || ws_bytes < need || !blast::aligned(ws, 16))) return BLAST_ERR_WORKSPACE;
  a.part = static_cast<float*>(ws);
  a.h = h_out;
  a.ldh = ldho;
  a.h_bf16 = h_dtype == BLAST_BF16;
  a.dx = dx;
  a.lddx = lddx;
  a.dx_bf16 = dx_dtype == BLAST_BF16;
  a.dh_in = dh_out;
  a.lddh_in = lddho;
  a.dh = dh;
  a.lddh = lddh;
  a.stats_in = stats;
  bool vec = params_pieces_ok(a) && pieces_ok(h_out, ldho, h_dtype) && pieces_ok(dx, lddx, dx_dtype) &&
             pieces_ok(dh_out, lddho, h_dtype) && pieces_ok(dh, lddh, h_dtype);
  if (branch) {
    a.y = y;
    a.ldy = ldy;
    a.y_bf16 = y_dtype == BLAST_BF16;
    a.dy = dy;
    a.lddy = lddy;
    a.dy_bf16 = dy_dtype == BLAST_BF16;
    vec = vec && pieces_ok(y, ldy, y_dtype) && pieces_ok(dy, lddy, dy_dtype);
    if (dgate && !gate_sum) {
      a.dgate = dgate;
      a.lddg = lddg;
      vec = vec && pieces_ok(dgate, lddg, P->g_dtype);
    }
  }
  return a.layer ? blast::norm_backward_layer(a, vec, stream) : blast::norm_backward_rms(a, vec, stream);
}
