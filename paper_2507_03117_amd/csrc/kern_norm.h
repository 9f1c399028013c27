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
  const int64_t t = (int64_t)blockIdx.x * ROWS + (NW == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);
  if (t >= a.T) return;  // (whole waves; with NW > 1 whole workgroups)
  RowSum<NW> row_sum{red, (int)(threadIdx.x >> 6)};
  const int E = a.width;
  const float inv_e = 1.0f / (float)E;
  const bool branch = a.y != nullptr;
  auto ask = [&](Piece (&q)[NCH], const void* p, int64_t at, int bf16) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      q[c] = Piece{};
      if (p) piece_load<NT, VEC>(q[c], row_of(p, at, bf16), c, lane, E, bf16);
    }
  };
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
  Piece h[NCH], g[NCH], w[NCH], b[NCH];
  if (branch) {
    Piece y[NCH], pw[NCH], pb[NCH];
    float p[NCH][8];
    ask(y, a.y, t * a.ldy, a.y_bf16);
    ask(h, a.h, t * a.ldh, a.h_bf16);
    ask(g, a.gate, t * a.ldg, a.g_bf16);
    ask(pw, a.pw, 0, a.p_bf16);
    ask(pb, a.pb, 0, a.p_bf16);
#pragma unroll
    for (int c = 0; c < NCH; ++c) piece_values<VEC>(y[c], a.y_bf16, p[c]);
    if (a.post) {
      normalise(p, st[2], st[3]);
#pragma unroll
      for (int c = 0; c < NCH; ++c) affine(p[c], pw[c], a.pw != nullptr, pb[c], a.pb != nullptr);
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      piece_values<VEC>(h[c], a.h_bf16, v[c]);
      if (a.gate) {
        float f[8];
        piece_values<VEC>(g[c], a.g_bf16, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) p[c][j] *= f[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[c][j] = __builtin_fmaf(a.scale, p[c][j], v[c][j]);
      piece_store<NT, VEC>(row_of(a.h_out, t * a.ldho, a.h_bf16), c, lane, E, a.h_bf16, v[c]);
    }
  } else {
    ask(h, a.h, t * a.ldh, a.h_bf16);
  }
  // (in registers that the branch no longer needs; the row's sums take a while)
  ask(w, a.w, 0, a.p_bf16);
  ask(b, a.b, 0, a.p_bf16);
  if (!branch) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) piece_values<VEC>(h[c], a.h_bf16, v[c]);
  }
  normalise(v, st[0], st[1]);
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    affine(v[c], w[c], a.w != nullptr, b[c], a.b != nullptr);
    piece_store<NT, VEC>(row_of(a.x, t * a.ldx, a.x_bf16), c, lane, E, a.x_bf16, v[c]);
  }
  if (a.stats && lane == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a.stats[t * 4 + i] = st[i];
  }
}

// The gradient.  A workgroup holds TEAMS rows at a time, NW waves to a row, and goes over its share of the rows with the
// columns' sums kept per lane: in registers, the first NL of them (dweight first) in LDS where a row leaves no registers for
// them.  MODE: 0 no branch, 1 branch without a norm of its own, 2 with one.  LOW: every operand is bf16, whose pieces take half the
// registers.
template <int NW, int NCH, int TEAMS, bool VEC, bool LAYER, int MODE, int NL, bool LOW>
__global__ __launch_bounds__(64 * NW * TEAMS) void k_norm_backward(const NormArgs a) {
  static_assert(NL == 0 || TEAMS == 1, "sums in LDS are one row's");
  constexpr int NT = 64 * NW;
  const int h_bf16 = LOW ? 1 : a.h_bf16, y_bf16 = LOW ? 1 : a.y_bf16, g_bf16 = LOW ? 1 : a.g_bf16, p_bf16 = LOW ? 1 : a.p_bf16;
  const int dx_bf16 = LOW ? 1 : a.dx_bf16, dy_bf16 = LOW ? 1 : a.dy_bf16;
  // column sums: dweight | dgate | dpost_weight | dbias | dpost_bias, those that MODE and LAYER know
  constexpr bool kSum[kNormSums] = {true, MODE >= 1, MODE == 2, LAYER, LAYER && MODE == 2};
  constexpr int kInLds[kNormSums] = {NL > 0 ? 0 : -1, -1, NL > 1 ? 1 : -1, -1, -1};
  __shared__ float red[TEAMS][2][NW][2];
  extern __shared__ __attribute__((aligned(16))) float pool[];  // sums in LDS [NL][NCH][2][NT][4], or where the teams' sums meet
  const int team = TEAMS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT), lane = TEAMS == 1 ? threadIdx.x : threadIdx.x % NT;
  RowSum<NW> row_sum{red[team], lane >> 6};
  const int E = a.width;
  const float inv_e = 1.0f / (float)E;
  float sum[kNormSums][NCH][8];
#pragma unroll
  for (int s = 0; s < kNormSums; ++s)
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[s][c][j] = 0.0f;
  auto slot = [&](int s, int c, int half) { return reinterpret_cast<float4*>(pool) + ((kInLds[s] * NCH + c) * 2 + half) * NT + lane; };
  if constexpr (NL > 0) {
#pragma unroll
    for (int s = 0; s < kNormSums; ++s)
#pragma unroll
      for (int c = 0; c < NCH; ++c)
        if (kInLds[s] >= 0) *slot(s, c, 0) = *slot(s, c, 1) = float4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // adds a piece's terms u v (or u alone) to sum s
  auto accumulate = [&](auto s, int c, const float (&u)[8], const float (&v)[8]) {
    if constexpr (kInLds[s.value] >= 0) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float4* q = slot(s.value, c, half);
        float4 t = *q;
        t.x = __builtin_fmaf(u[4 * half], v[4 * half], t.x);
        t.y = __builtin_fmaf(u[4 * half + 1], v[4 * half + 1], t.y);
        t.z = __builtin_fmaf(u[4 * half + 2], v[4 * half + 2], t.z);
        t.w = __builtin_fmaf(u[4 * half + 3], v[4 * half + 3], t.w);
        *q = t;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[s.value][c][j] = __builtin_fmaf(u[j], v[j], sum[s.value][c][j]);
    }
  };
  auto inside = [&](int c, int j) { return piece_at<NT, VEC>(c, j, lane) < E; };
  // gradient of the values a norm was taken of: d (that of the normalised ones n) -> r (d - n mean(d n) - mean(d))
  auto through = [&](float (&d)[NCH][8], const float (&n)[NCH][8], float r) {
    float s[LAYER ? 2 : 1] = {};
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s[0] = __builtin_fmaf(d[c][j], n[c][j], s[0]);
        if constexpr (LAYER) s[1] += d[c][j];
      }
    row_sum(s);
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float v = __builtin_fmaf(-n[c][j], s[0] * inv_e, d[c][j]);
        if constexpr (LAYER) v -= s[1] * inv_e;
        d[c][j] = r * v;
      }
  };
  auto times = [&](float (&v)[8], const void* p, const Piece& q, int bf16) {
    if (p) {
      float f[8];
      piece_values<VEC>(q, bf16, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= f[j];
    }
  };
  using S0 = std::integral_constant<int, 0>;
  using S2 = std::integral_constant<int, 2>;
  for (int64_t first = (int64_t)blockIdx.x * TEAMS; first < a.T; first += (int64_t)gridDim.x * TEAMS) {
    // (a team without a row goes along on the last one, for the barriers, and keeps nothing)
    const bool mine = TEAMS == 1 || first + team < a.T;
    const int64_t t = mine ? first + team : a.T - 1;
    float d[NCH][8], n[NCH][8];
    const float4 st = scalar_float4(a.stats_in + t * 4);
    Piece dhi[NCH], y[NCH], g[NCH], pw[NCH], pb[NCH];
    {
      Piece h[NCH], dx[NCH], w[NCH];
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        h[c] = dx[c] = w[c] = Piece{};
        piece_load<NT, VEC>(h[c], row_of(a.h, t * a.ldh, h_bf16), c, lane, E, h_bf16);
        piece_load<NT, VEC>(dx[c], row_of(a.dx, t * a.lddx, dx_bf16), c, lane, E, dx_bf16);
        if (a.w) piece_load<NT, VEC>(w[c], row_of(a.w, 0, p_bf16), c, lane, E, p_bf16);
      }
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        dhi[c] = y[c] = Piece{};
        if (a.dh_in) piece_load<NT, VEC>(dhi[c], row_of(a.dh_in, t * a.lddh_in, h_bf16), c, lane, E, h_bf16);
        if constexpr (MODE >= 1) piece_load<NT, VEC>(y[c], row_of(a.y, t * a.ldy, y_bf16), c, lane, E, y_bf16);
      }
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        piece_values<VEC>(h[c], h_bf16, n[c]);
        piece_values<VEC>(dx[c], dx_bf16, d[c]);
#pragma unroll
        for (int j = 0; j < 8; ++j) n[c][j] = inside(c, j) ? (n[c][j] - st.x) * st.y : 0.0f;
        if (mine) {
          accumulate(S0{}, c, d[c], n[c]);
          if constexpr (LAYER) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[3][c][j] += d[c][j];
          }
        }
        times(d[c], a.w, w[c], p_bf16);
      }
    }
    // (what the branch needs is asked for here: its registers were the stream's until now, and the row's sums take a while)
    if constexpr (MODE >= 1) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        g[c] = Piece{};
        if (a.gate) piece_load<NT, VEC>(g[c], row_of(a.gate, t * a.ldg, g_bf16), c, lane, E, g_bf16);
        if constexpr (MODE == 2) {
          pw[c] = pb[c] = Piece{};
          if (a.pw) piece_load<NT, VEC>(pw[c], row_of(a.pw, 0, p_bf16), c, lane, E, p_bf16);
          if (LAYER && a.pb) piece_load<NT, VEC>(pb[c], row_of(a.pb, 0, p_bf16), c, lane, E, p_bf16);
        }
      }
    }
    through(d, n, st.y);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (a.dh_in) {
        float f[8];
        piece_values<VEC>(dhi[c], h_bf16, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[c][j] += f[j];
      }
      if (mine) piece_store<NT, VEC>(row_of(a.dh, t * a.lddh, h_bf16), c, lane, E, h_bf16, d[c]);
    }
    if constexpr (MODE >= 1) {
      // d: gradient of the stream.  n: y, or its normalised values
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        float p[8];
        piece_values<VEC>(y[c], y_bf16, n[c]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (MODE == 2) n[c][j] = inside(c, j) ? (n[c][j] - st.z) * st.w : 0.0f;
          p[j] = n[c][j];
          d[c][j] = inside(c, j) ? d[c][j] * a.scale : 0.0f;
        }
        if (a.gate) {
          if constexpr (MODE == 2) {
            times(p, a.pw, pw[c], p_bf16);
            if (LAYER && a.pb) {
              float f[8];
              piece_values<VEC>(pb[c], p_bf16, f);
#pragma unroll
              for (int j = 0; j < 8; ++j) p[j] += f[j];
            }
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) p[j] *= d[c][j];
          times(d[c], a.gate, g[c], g_bf16);
          if (mine) {
            if (a.ldg == 0) {
#pragma unroll
              for (int j = 0; j < 8; ++j) sum[1][c][j] += p[j];
            } else if (a.dgate) {
              piece_store<NT, VEC>(row_of(a.dgate, t * a.lddg, g_bf16), c, lane, E, g_bf16, p);
            }
          }
        }
        if constexpr (MODE == 2) {
          if (mine) {
            accumulate(S2{}, c, d[c], n[c]);
            if constexpr (LAYER) {
#pragma unroll
              for (int j = 0; j < 8; ++j) sum[4][c][j] += d[c][j];
            }
          }
          times(d[c], a.pw, pw[c], p_bf16);
        }
      }
      if constexpr (MODE == 2) through(d, n, st.w);
      if (a.dy && mine) {
#pragma unroll
        for (int c = 0; c < NCH; ++c) piece_store<NT, VEC>(row_of(a.dy, t * a.lddy, dy_bf16), c, lane, E, dy_bf16, d[c]);
      }
    }
  }
  // ---- the workgroup's column sums
  float* out = a.part;
#pragma unroll
  for (int s = 0; s < kNormSums; ++s) {
    if (!kSum[s] || !a.sum_out[s]) continue;
    float* dst = gridDim.x == 1 ? a.sum_out[s] : out + (int64_t)blockIdx.x * E;
    out += (int64_t)gridDim.x * E;
    if constexpr (TEAMS > 1) {
      __syncthreads();
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) pool[team * (NT * NCH * 8) + piece_at<NT, VEC>(c, j, lane)] = sum[s][c][j];
      __syncthreads();
      for (int e = threadIdx.x; e < E; e += NT * TEAMS) {
        float v = pool[e];
#pragma unroll
        for (int k = 1; k < TEAMS; ++k) v += pool[k * (NT * NCH * 8) + e];
        dst[e] = v;
      }
    } else {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        if constexpr (NL > 0) {
          if (kInLds[s] >= 0) {
            const float4 lo = *slot(s, c, 0), hi = *slot(s, c, 1);
            const float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[s][c][j] = v[j];
          }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int e = piece_at<NT, VEC>(c, j, lane);
          if (e < E) dst[e] = sum[s][c][j];
        }
      }
    }
  }
}

}  // namespace blast_dev
