// The step between two blocks of a residual network and its gradient: gated residual add, norm of the branch, norm of the
// stream (formulas: blast_norm_residual, blast_norm_residual_backward in blast.h).
//
// Bound: memory.  Forward, every input is read and every output written once; backward too, and the column sums (gradients
// of the weights) stay in the registers of the lanes that own the columns while a workgroup goes over its rows.  A row is
// held in the registers of NW waves, NCH pieces of eight values to a lane, so that the variance is taken of the centred values
// without a second read; sums over a row are DPP steps and, for NW > 1, one barrier.  With NW = 1 the workgroup's four waves
// have a row each and no barrier.
#pragma once
#include "kern_rows.h"

namespace blast_dev {

struct NormArgs {
  const void *h, *y, *gate, *w, *b, *pw, *pb, *dx, *dh_in;
  const float* stats_in;
  void *h_out, *x, *dh, *dy, *dgate;
  float* stats;
  float* part;  // column sums of the workgroups, [sum][workgroup][width]; with one workgroup the sums themselves
  float* sum_out[5];  // slots: dweight, dgate, dpost_weight, dbias, dpost_bias (null: not wanted)
  int64_t ldh, ldy, ldg, ldho, ldx, lddx, lddh_in, lddh, lddy, lddg;
  int64_t T;
  int width;
  int h_bf16, y_bf16, g_bf16, p_bf16, x_bf16, dx_bf16, dy_bf16;
  int layer, post;
  float eps, scale;
};

constexpr int kNormSums = 5;

template <int NW, int NCH, bool VEC>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW) void k_norm_residual(const NormArgs a) {
  constexpr int NT = 64 * NW, ROWS = NW == 1 ? 4 : 1;
  __shared__ float red[2][NW][2];
  const int lane = NW == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t t = (int64_t)blockIdx.x * ROWS + (NW == 1 ? threadIdx.x >> 6 : 0);
  if (t >= a.T) return;  // (whole waves; with NW > 1 whole workgroups)
  RowSum<NW> row_sum{red};
  const int E = a.width;
  const float inv_e = 1.0f / (float)E;
  const bool branch = a.y != nullptr;
  Piece h[NCH], y[NCH], g[NCH], w[NCH], b[NCH], pw[NCH], pb[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    h[c] = y[c] = g[c] = w[c] = b[c] = pw[c] = pb[c] = Piece{};
    piece_load<NT, VEC>(h[c], a.h, t * a.ldh, c, lane, E, a.h_bf16);
    if (branch) piece_load<NT, VEC>(y[c], a.y, t * a.ldy, c, lane, E, a.y_bf16);
    if (a.gate) piece_load<NT, VEC>(g[c], a.gate, t * a.ldg, c, lane, E, a.g_bf16);
    if (a.w) piece_load<NT, VEC>(w[c], a.w, 0, c, lane, E, a.p_bf16);
    if (a.b) piece_load<NT, VEC>(b[c], a.b, 0, c, lane, E, a.p_bf16);
    if (a.pw) piece_load<NT, VEC>(pw[c], a.pw, 0, c, lane, E, a.p_bf16);
    if (a.pb) piece_load<NT, VEC>(pb[c], a.pb, 0, c, lane, E, a.p_bf16);
  }
  auto inside = [&](int c, int j) { return piece_at<NT, VEC>(c, j, lane) < E; };
  // mean (0 without `layer`) and reciprocal deviation; v becomes the normalised values
  auto normalise = [&](float (&v)[NCH][8], float& mean, float& r) {
    mean = 0.0f;
    if (a.layer) {
      float s[1] = {0.0f};
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] += v[c][j];
      row_sum(s);
      mean = s[0] * inv_e;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] = inside(c, j) ? v[c][j] - mean : 0.0f;
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) s[0] = __builtin_fmaf(v[c][j], v[c][j], s[0]);
    row_sum(s);
    r = rsqrtf(s[0] * inv_e + a.eps);
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[c][j] *= r;
  };
  auto affine = [&](float (&v)[8], const Piece& weight, bool has_weight, const Piece& bias, bool has_bias) {
    float f[8];
    if (has_weight) {
      piece_values<VEC>(weight, a.p_bf16, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= f[j];
    }
    if (has_bias) {
      piece_values<VEC>(bias, a.p_bf16, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += f[j];
    }
  };
  float v[NCH][8], st[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int c = 0; c < NCH; ++c) piece_values<VEC>(h[c], a.h_bf16, v[c]);
  if (branch) {
    float p[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c) piece_values<VEC>(y[c], a.y_bf16, p[c]);
    if (a.post) {
      normalise(p, st[2], st[3]);
#pragma unroll
      for (int c = 0; c < NCH; ++c) affine(p[c], pw[c], a.pw != nullptr, pb[c], a.pb != nullptr);
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (a.gate) {
        float f[8];
        piece_values<VEC>(g[c], a.g_bf16, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) p[c][j] *= f[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[c][j] = __builtin_fmaf(a.scale, p[c][j], v[c][j]);
      piece_store<NT, VEC>(a.h_out, t * a.ldho, c, lane, E, a.h_bf16, v[c]);
    }
  }
  normalise(v, st[0], st[1]);
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    affine(v[c], w[c], a.w != nullptr, b[c], a.b != nullptr);
    piece_store<NT, VEC>(a.x, t * a.ldx, c, lane, E, a.x_bf16, v[c]);
  }
  if (a.stats && lane == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a.stats[t * 4 + i] = st[i];
  }
}

// MODE: 0 no branch, 1 branch without a norm of its own, 2 with one.
template <int NW, int NCH, bool VEC, bool LAYER, int MODE>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW) void k_norm_backward(const NormArgs a) {
  constexpr int NT = 64 * NW, ROWS = NW == 1 ? 4 : 1;
  // column sums of this workgroup's rows: dweight | dgate | dpost_weight | dbias | dpost_bias, those that MODE and LAYER know
  constexpr bool kSum[kNormSums] = {true, MODE >= 1, MODE == 2, LAYER, LAYER && MODE == 2};
  __shared__ float red[2][NW][2];
  const int lane = NW == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int team = NW == 1 ? threadIdx.x >> 6 : 0;
  RowSum<NW> row_sum{red};
  const int E = a.width;
  const float inv_e = 1.0f / (float)E;
  float sum[kNormSums][NCH][8];
#pragma unroll
  for (int s = 0; s < kNormSums; ++s)
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[s][c][j] = 0.0f;
  auto inside = [&](int c, int j) { return piece_at<NT, VEC>(c, j, lane) < E; };
  // gradient of the values a norm was taken of: d (that of the normalised ones n) -> r (d - n mean(d n) - mean(d))
  auto through = [&](float (&d)[NCH][8], const float (&n)[NCH][8], float r) {
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s[0] = __builtin_fmaf(d[c][j], n[c][j], s[0]);
        if (LAYER) s[1] += d[c][j];
      }
    if constexpr (LAYER) {
      row_sum(s);
    } else {
      float one[1] = {s[0]};
      row_sum(one);
      s[0] = one[0];
    }
    s[0] *= inv_e;
    s[1] *= inv_e;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float v = __builtin_fmaf(-n[c][j], s[0], d[c][j]);
        if (LAYER) v -= s[1];
        d[c][j] = r * v;
      }
  };
  for (int64_t t = (int64_t)blockIdx.x * ROWS + team; t < a.T; t += (int64_t)gridDim.x * ROWS) {
    Piece h[NCH], dx[NCH], dhi[NCH], y[NCH], g[NCH], w[NCH], pw[NCH], pb[NCH];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      h[c] = dx[c] = dhi[c] = y[c] = g[c] = w[c] = pw[c] = pb[c] = Piece{};
      piece_load<NT, VEC>(h[c], a.h, t * a.ldh, c, lane, E, a.h_bf16);
      piece_load<NT, VEC>(dx[c], a.dx, t * a.lddx, c, lane, E, a.dx_bf16);
      if (a.dh_in) piece_load<NT, VEC>(dhi[c], a.dh_in, t * a.lddh_in, c, lane, E, a.h_bf16);
      if (a.w) piece_load<NT, VEC>(w[c], a.w, 0, c, lane, E, a.p_bf16);
      if constexpr (MODE >= 1) {
        piece_load<NT, VEC>(y[c], a.y, t * a.ldy, c, lane, E, a.y_bf16);
        if (a.gate) piece_load<NT, VEC>(g[c], a.gate, t * a.ldg, c, lane, E, a.g_bf16);
      }
      if constexpr (MODE == 2) {
        if (a.pw) piece_load<NT, VEC>(pw[c], a.pw, 0, c, lane, E, a.p_bf16);
        if (a.pb) piece_load<NT, VEC>(pb[c], a.pb, 0, c, lane, E, a.p_bf16);
      }
    }
    const float4 st = *reinterpret_cast<const float4*>(a.stats_in + t * 4);
    float d[NCH][8], n[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      float f[8];
      piece_values<VEC>(h[c], a.h_bf16, n[c]);
      piece_values<VEC>(dx[c], a.dx_bf16, d[c]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        n[c][j] = inside(c, j) ? (n[c][j] - st.x) * st.y : 0.0f;
        sum[0][c][j] = __builtin_fmaf(d[c][j], n[c][j], sum[0][c][j]);
        if (LAYER) sum[3][c][j] += d[c][j];
      }
      if (a.w) {
        piece_values<VEC>(w[c], a.p_bf16, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[c][j] *= f[j];
      }
    }
    through(d, n, st.y);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (a.dh_in) {
        float f[8];
        piece_values<VEC>(dhi[c], a.h_bf16, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[c][j] += f[j];
      }
      piece_store<NT, VEC>(a.dh, t * a.lddh, c, lane, E, a.h_bf16, d[c]);
    }
    if constexpr (MODE >= 1) {
      // d: gradient of the stream.  n: y, or its normalised values
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        float f[8], p[8];
        piece_values<VEC>(y[c], a.y_bf16, n[c]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (MODE == 2) n[c][j] = inside(c, j) ? (n[c][j] - st.z) * st.w : 0.0f;
          p[j] = n[c][j];
          d[c][j] = inside(c, j) ? d[c][j] * a.scale : 0.0f;
        }
        if constexpr (MODE == 2) {
          if (a.pw) {
            piece_values<VEC>(pw[c], a.p_bf16, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] *= f[j];
          }
          if (a.pb) {
            piece_values<VEC>(pb[c], a.p_bf16, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] += f[j];
          }
        }
        if (a.gate) {
          piece_values<VEC>(g[c], a.g_bf16, f);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            p[j] *= d[c][j];
            d[c][j] *= f[j];
          }
          if (a.ldg == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[1][c][j] += p[j];
          } else if (a.dgate) {
            piece_store<NT, VEC>(a.dgate, t * a.lddg, c, lane, E, a.g_bf16, p);
          }
        }
        if constexpr (MODE == 2) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            sum[2][c][j] = __builtin_fmaf(d[c][j], n[c][j], sum[2][c][j]);
            if (LAYER) sum[4][c][j] += d[c][j];
          }
          if (a.pw) {
            piece_values<VEC>(pw[c], a.p_bf16, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) d[c][j] *= f[j];
          }
        }
      }
      if constexpr (MODE == 2) through(d, n, st.w);
      if (a.dy) {
#pragma unroll
        for (int c = 0; c < NCH; ++c) piece_store<NT, VEC>(a.dy, t * a.lddy, c, lane, E, a.dy_bf16, d[c]);
      }
    }
  }
  // ---- the workgroup's column sums
  __shared__ float join[NW == 1 ? 4 : 1][NW == 1 ? NCH * 512 : 1];
  float* out = a.part;
#pragma unroll
  for (int s = 0; s < kNormSums; ++s) {
    if (!kSum[s] || !a.sum_out[s]) continue;
    float* dst = gridDim.x == 1 ? a.sum_out[s] : out + (int64_t)blockIdx.x * E;
    out += (int64_t)gridDim.x * E;
    if constexpr (NW == 1) {
      __syncthreads();
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) join[team][piece_at<NT, VEC>(c, j, lane)] = sum[s][c][j];
      __syncthreads();
      for (int e = threadIdx.x; e < E; e += 256) dst[e] = (join[0][e] + join[1][e]) + (join[2][e] + join[3][e]);
    } else {
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int e = piece_at<NT, VEC>(c, j, lane);
          if (e < E) dst[e] = sum[s][c][j];
        }
    }
  }
}

}  // namespace blast_dev
