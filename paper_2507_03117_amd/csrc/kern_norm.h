// The step between two blocks of a residual network and its gradient: gated residual add, norm of the branch, norm of the
// stream (formulas: blast_norm_residual, blast_norm_residual_backward in blast.h).
//
// Bound: memory.  Forward, every input is read and every output written once; backward too, and the column sums (gradients
// of the weights) stay with the lanes that own the columns while a workgroup goes over its rows.  A row is held in the
// registers of NW waves, NCH pieces of eight values to a lane, so that the variance is taken of the centred values without a second
// read; sums over a row are DPP steps and, for NW > 1, one barrier.  With NW = 1 a forward workgroup's four waves have a row each
// and no barrier.  Why one piece a lane up to 8192 features: four waves of one piece against two of two, 2048 features, 4096 rows
// 13.2 / 13.8 us, forward, 1600 features, 333 rows 3.7 / 4.7.  Row addresses are scalar with one 32-bit offset a lane: 64-bit addresses
// of a dozen tensors took 39 registers more (the gradient of 2048 features, RMS on both sides, has 107).
// Measured, a launch among others in a recorded graph (by itself in a kernel trace it takes 0.5 to 1 us more; a copy of 1 GB moves
// 5.0 TB/s, of 64 MB in the last-level cache 7.8): forward, 2048 x 2048, norms on both sides, fp32 stream 11.9 us (4.2 TB/s); 4096 x
// 4096, bf16 24.3 (5.5); 2048 x 16384, gate per token 66.6 (5.0); 333 x 1600 3.7; one row of 4096, in a trace 2.9.  Gradient, with
// the launch that joins the sums: 2048 x 2048 20.1 us (3.8), 4096 x 4096 48.8 (4.1), 2048 x 16384 118 (4.6), 333 x 1600 6.8, 16 x 4096 3.5.
#pragma once
#include "kern_rows.h"

namespace blast_dev {

struct NormArgs {
  const void *h, *y, *gate, *w, *b, *pw, *pb, *dx, *dh_in;
  const float* stats_in;
  void *h_out, *x, *dh, *dy, *dgate;
  float* stats;
  float* part;  // column sums of the workgroups, [sum wanted][workgroup][width] (one workgroup writes sum_out instead)
  float* sum_out[5];  // dweight, dbias, dgate of one row, dpost_weight, dpost_bias (null: not wanted)
  int64_t ldh, ldy, ldg, ldho, ldx, lddx, lddh_in, lddh, lddy, lddg;
  int64_t T;
  int width;
  int h_bf16, y_bf16, g_bf16, p_bf16, x_bf16, dx_bf16, dy_bf16;
  int layer, post;
  float eps, scale;
  int column_groups;  // workgroups of a gradient launch that own columns (see norm_columns)
  int past;  // the stream's new values leave past the L2
};

// A stream of this size or more is written past the L2s (4 MB each, 32 together), which it would only empty: it is read again after
// the block's products.  4096 x 4096 bf16 26.2 -> 24.3 us, 2048 x 8192 31.7 -> 27.9, 2048 x 12000 fp32 107.5 -> 97.5, 2048 x 16384
// with a gate per token 66.3 -> 66.6; the step, two products and the next step with 4096 x 4096 141 -> 139.  Smaller streams gain alone
// (2048 x 4096 bf16 13.2 -> 12.4) and lose in that chain (78.6 -> 82.0), as x and the gradients do, which the next launch reads.
constexpr int64_t kPastBytes = 32 << 20;

constexpr int kNormSums = 5;

// LOOP: a workgroup goes over its share of the rows, else it has one.  AHEAD, LOW: see the gradient.
template <int NW, int NCH, bool VEC, bool LOOP, bool AHEAD, bool LOW>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW) void k_norm_residual(const NormArgs a) {
  constexpr int NT = 64 * NW, ROWS = NW == 1 ? 4 : 1;
  const int h_bf16 = LOW ? 1 : a.h_bf16, y_bf16 = LOW ? 1 : a.y_bf16, g_bf16 = LOW ? 1 : a.g_bf16, p_bf16 = LOW ? 1 : a.p_bf16;
  __shared__ float red[2][NW][2];
  const int lane = NW == 1 ? threadIdx.x & 63 : threadIdx.x;
  RowSum<NW> row_sum{red, (int)(threadIdx.x >> 6)};
  const int E = a.width;
  const float inv_e = 1.0f / (float)E;
  const bool branch = a.y != nullptr;
  auto ask = [&](Piece (&q)[NCH], const void* p, int64_t at, int bf16, bool fresh) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (fresh) q[c] = Piece{};
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
      piece_values<VEC>(weight, p_bf16, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= f[j];
    }
    if (has_bias) {
      piece_values<VEC>(bias, p_bf16, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += f[j];
    }
  };
  const int64_t step = (int64_t)gridDim.x * ROWS;
  int64_t t = (int64_t)blockIdx.x * ROWS + (NW == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);
  Piece h[NCH], y[NCH], g[NCH];
  auto ask_row = [&](int64_t row, bool fresh) {
    ask(y, a.y, row * a.ldy, y_bf16, fresh);
    ask(h, a.h, row * a.ldh, h_bf16, fresh);
    ask(g, a.gate, row * a.ldg, g_bf16, fresh);
  };
  if (t >= a.T) return;  // (with NW > 1 the whole workgroup has the row)
  if (AHEAD) ask_row(t, true);
  auto row = [&]() {
    const bool more = AHEAD && t + step < a.T;
    if (!AHEAD) ask_row(t, true);
    float v[NCH][8], st[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    Piece w[NCH], b[NCH];
    if (branch) {
      Piece pw[NCH], pb[NCH];
      float p[NCH][8];
      ask(pw, a.pw, 0, p_bf16, true);
      ask(pb, a.pb, 0, p_bf16, true);
#pragma unroll
      for (int c = 0; c < NCH; ++c) piece_values<VEC>(y[c], y_bf16, p[c]);
      if (more) ask(y, a.y, (t + step) * a.ldy, y_bf16, false);
      if (a.post) {
        normalise(p, st[2], st[3]);
#pragma unroll
        for (int c = 0; c < NCH; ++c) affine(p[c], pw[c], a.pw != nullptr, pb[c], a.pb != nullptr);
      }
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        piece_values<VEC>(h[c], h_bf16, v[c]);
        if (a.gate) {
          float f[8];
          piece_values<VEC>(g[c], g_bf16, f);
#pragma unroll
          for (int j = 0; j < 8; ++j) p[c][j] *= f[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] = __builtin_fmaf(a.scale, p[c][j], v[c][j]);
        unsigned char* to = row_of(a.h_out, t * a.ldho, h_bf16);
        if (a.past)
          piece_store<NT, VEC, true>(to, c, lane, E, h_bf16, v[c]);
        else
          piece_store<NT, VEC>(to, c, lane, E, h_bf16, v[c]);
      }
      if (more) ask(g, a.gate, (t + step) * a.ldg, g_bf16, false);
    } else {
#pragma unroll
      for (int c = 0; c < NCH; ++c) piece_values<VEC>(h[c], h_bf16, v[c]);
    }
    if (more) ask(h, a.h, (t + step) * a.ldh, h_bf16, false);
    // (in registers that the branch no longer needs; the row's sums take a while)
    ask(w, a.w, 0, p_bf16, true);
    ask(b, a.b, 0, p_bf16, true);
    normalise(v, st[0], st[1]);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      affine(v[c], w[c], a.w != nullptr, b[c], a.b != nullptr);
      piece_store<NT, VEC>(row_of(a.x, t * a.ldx, a.x_bf16), c, lane, E, a.x_bf16, v[c]);
    }
    if (a.stats && lane == 0) *reinterpret_cast<float4*>(a.stats + t * 4) = float4{st[0], st[1], st[2], st[3]};
  };
  if constexpr (LOOP) {
    for (; t < a.T; t += step) row();
  } else {
    row();
  }
}

// dweight and dbias of 32 columns over all rows: they need the statistics but no sum over a row, so that workgroups beside
// those of the rows can have them, in the same launch, where there are few rows.  Four lanes to a row, two rows of a lane on
// their way at a time; two neighbouring workgroups of an XCD (ids eight apart) share the 128-byte lines of bf16.
constexpr int kNormOwned = 32;
template <int THREADS, bool VEC, bool LAYER>
__device__ __forceinline__ void norm_columns(const NormArgs& a, int id) {
  constexpr int kLanes = kNormOwned / 8, kRows = THREADS / kLanes, kWaves = THREADS / 64;
  __shared__ float red[kWaves][kNormOwned];
  const int lane = threadIdx.x % kLanes, team = threadIdx.x / kLanes;
  const int col0 = ((id / 16) * 16 + (id % 8) * 2 + id / 8 % 2) * kNormOwned;
  const int width = a.width - col0 < kNormOwned ? a.width - col0 : kNormOwned;
  if (width <= 0) return;
  float sum[2][8];
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[0][j] = sum[1][j] = 0.0f;
  struct Row {
    Piece h, dx;
    float2 st;
  };
  auto read = [&](Row& q, int t) {
    q.h = q.dx = Piece{};
    piece_load<kLanes, VEC>(q.h, row_of(a.h, t * a.ldh + col0, a.h_bf16), 0, lane, width, a.h_bf16);
    piece_load<kLanes, VEC>(q.dx, row_of(a.dx, t * a.lddx + col0, a.dx_bf16), 0, lane, width, a.dx_bf16);
    q.st = *reinterpret_cast<const float2*>(a.stats_in + (int64_t)t * 4);
  };
  auto add = [&](const Row& q) {
    float n[8], d[8];
    piece_values<VEC>(q.h, a.h_bf16, n);
    piece_values<VEC>(q.dx, a.dx_bf16, d);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sum[0][j] = __builtin_fmaf(d[j], (n[j] - q.st.x) * q.st.y, sum[0][j]);
      if (LAYER) sum[1][j] += d[j];
    }
  };
  for (int t = team; t < a.T; t += 2 * kRows) {
    Row q0, q1;
    read(q0, t);
    const bool two = t + kRows < a.T;
    if (two) read(q1, t + kRows);
    add(q0);
    if (two) add(q1);
  }
  // the sixteen rows of a wave, then the waves in order
#pragma unroll
  for (int s = 0; s < (LAYER ? 2 : 1); ++s) {
    if (!a.sum_out[s]) continue;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float v = sum[s][j];
#pragma unroll
      for (int m = kLanes; m < 64; m *= 2) v += __shfl_xor(v, m);
      if ((threadIdx.x & 63) < kLanes) red[threadIdx.x >> 6][piece_at<kLanes, VEC>(0, j, lane)] = v;
    }
    __syncthreads();
    const int e = threadIdx.x;
    if (e < width) {
      float v = red[0][e];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += red[w][e];
      a.sum_out[s][col0 + e] = v;
    }
  }
}

// The gradient.  A workgroup holds TEAMS rows at a time, NW waves to a row, and goes over its share of the rows.  Over the
// rows it keeps at most four sums per column, whatever is wanted of the branch:
//     dx n (dweight),  dx (dbias),  q m,  q      with q = dh, times the gate where that has a row per token;
// the gradients of a gate of one row, the branch's weight and its bias are those sums times factors of the column, applied at
// the end.  The first NL of them are in LDS (a lane's own slots), the others in registers.
// Rows one ahead (AHEAD): a tensor's registers take the next row's values as soon as this row's have been used, so that they
// arrive during this row's sums and stores.  LOW: every operand is bf16, whose pieces take half the registers.
// LOOP = false: a workgroup has its TEAMS rows and no others.  COLS: the first workgroups own columns instead, and the others keep
// no sums.  MODE: 0 no branch, 1 branch without a norm of its own, 2 with one.
template <int NW, int NCH, int TEAMS, bool VEC, bool LAYER, int MODE, int NL, bool LOOP, bool AHEAD, bool LOW, bool COLS>
__global__ __launch_bounds__(64 * NW * TEAMS) void k_norm_backward(const NormArgs a) {
  constexpr int NT = 64 * NW;
  static_assert(!COLS || (!LOOP && TEAMS == 1 && MODE < 2), "few rows, and sums that need no other over a row");
  if constexpr (COLS) {
    if ((int)blockIdx.x < a.column_groups) {
      norm_columns<NT, VEC, LAYER>(a, blockIdx.x);
      return;
    }
  }
  constexpr int kDw = 0, kQm = 1, kDx = 2, kQ = 3;
  constexpr bool kSum[4] = {true, MODE >= 1, LAYER, LAYER && MODE == 2};  // those that MODE and LAYER know
  constexpr int kOrder[4] = {0, MODE >= 1 ? 1 : -1, !LAYER ? -1 : MODE >= 1 ? 2 : 1, LAYER && MODE == 2 ? 3 : -1};
  constexpr auto in_lds = [](int s) { return kOrder[s] >= 0 && kOrder[s] < NL; };
  static_assert(TEAMS == 1 || NL >= kOrder[0] + 1 + (MODE >= 1) + LAYER + (LAYER && MODE == 2), "the teams' sums meet in LDS");
  const int h_bf16 = LOW ? 1 : a.h_bf16, y_bf16 = LOW ? 1 : a.y_bf16, g_bf16 = LOW ? 1 : a.g_bf16, p_bf16 = LOW ? 1 : a.p_bf16;
  const int dx_bf16 = LOW ? 1 : a.dx_bf16, dy_bf16 = LOW ? 1 : a.dy_bf16;
  __shared__ float red[TEAMS][2][NW][2];
  extern __shared__ __attribute__((aligned(16))) float pool[];  // [sum][NCH][2][lane of the workgroup][4]
  const int team = TEAMS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
  const int lane = TEAMS == 1 ? threadIdx.x : threadIdx.x % NT;
  RowSum<NW> row_sum{red[team], lane >> 6};
  const int E = a.width;
  const float inv_e = 1.0f / (float)E;
  float sum[4][NCH][8];
  auto slot = [&](int s, int c, int half, int of_team) {
    return reinterpret_cast<float4*>(pool) + ((kOrder[s] * NCH + c) * 2 + half) * (NT * TEAMS) + of_team * NT + lane;
  };
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[s][c][j] = 0.0f;
      if (in_lds(s)) *slot(s, c, 0, team) = *slot(s, c, 1, team) = float4{0.0f, 0.0f, 0.0f, 0.0f};
    }
  // adds a piece's terms u v (without `v`: u) to a sum
  auto accumulate = [&](auto which, int c, const float (&u)[8], const float (&v)[8]) {
    constexpr int s = which.value;
    constexpr bool plain = s == kDx || s == kQ;
    if constexpr (in_lds(s)) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float4* q = slot(s, c, half, team);
        float4 t = *q;
        const int o = 4 * half;
        t.x = plain ? t.x + u[o] : __builtin_fmaf(u[o], v[o], t.x);
        t.y = plain ? t.y + u[o + 1] : __builtin_fmaf(u[o + 1], v[o + 1], t.y);
        t.z = plain ? t.z + u[o + 2] : __builtin_fmaf(u[o + 2], v[o + 2], t.z);
        t.w = plain ? t.w + u[o + 3] : __builtin_fmaf(u[o + 3], v[o + 3], t.w);
        *q = t;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[s][c][j] = plain ? sum[s][c][j] + u[j] : __builtin_fmaf(u[j], v[j], sum[s][c][j]);
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
  auto plus = [&](float (&v)[8], const void* p, const Piece& q, int bf16) {
    if (p) {
      float f[8];
      piece_values<VEC>(q, bf16, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += f[j];
    }
  };
  auto ask = [&](Piece& q, const void* p, int64_t at, int c, int bf16) {
    if (!AHEAD) q = Piece{};  // (or what a row left in it would stay in registers until the next)
    if (p) piece_load<NT, VEC>(q, row_of(p, at, bf16), c, lane, E, bf16);
  };
  using Dw = std::integral_constant<int, kDw>;
  using Qm = std::integral_constant<int, kQm>;
  using Dx = std::integral_constant<int, kDx>;
  using Q = std::integral_constant<int, kQ>;
  const bool per_token = MODE >= 1 && a.gate && a.ldg != 0;
  const bool want_qm = a.sum_out[2] || a.sum_out[3], want_q = (a.sum_out[2] && a.pb) || a.sum_out[4];
  const int64_t step = (int64_t)gridDim.x * TEAMS;
  // (a team without a row goes along on the last one, for the barriers, and keeps nothing)
  auto row_at = [&](int64_t first) { return TEAMS == 1 || first + team < a.T ? first + team : a.T - 1; };
  Piece h[NCH], dx[NCH], dhi[NCH], y[NCH], g[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) h[c] = dx[c] = dhi[c] = y[c] = g[c] = Piece{};
  if constexpr (AHEAD) {
    const int64_t t = row_at((int64_t)blockIdx.x * TEAMS);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      ask(h[c], a.h, t * a.ldh, c, h_bf16);
      ask(dx[c], a.dx, t * a.lddx, c, dx_bf16);
      ask(dhi[c], a.dh_in, t * a.lddh_in, c, h_bf16);
      if constexpr (MODE >= 1) {
        ask(y[c], a.y, t * a.ldy, c, y_bf16);
        ask(g[c], a.gate, t * a.ldg, c, g_bf16);
      }
    }
  }
  auto rows = [&](int64_t first) {
    const bool mine = TEAMS == 1 || first + team < a.T, more = AHEAD && first + step < a.T;
    const int64_t t = row_at(first), next = more ? row_at(first + step) : t;
    float d[NCH][8], n[NCH][8];
    const float4 st = scalar_float4(a.stats_in + t * 4);
    Piece pw[NCH], pb[NCH];
    {
      Piece w[NCH];
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        if constexpr (!AHEAD) {
          ask(h[c], a.h, t * a.ldh, c, h_bf16);
          ask(dx[c], a.dx, t * a.lddx, c, dx_bf16);
        }
        w[c] = Piece{};
        ask(w[c], a.w, 0, c, p_bf16);
      }
      if constexpr (!AHEAD && NCH == 1) {
        ask(dhi[0], a.dh_in, t * a.lddh_in, 0, h_bf16);
        if constexpr (MODE >= 1) ask(y[0], a.y, t * a.ldy, 0, y_bf16);
      }
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        piece_values<VEC>(h[c], h_bf16, n[c]);
        piece_values<VEC>(dx[c], dx_bf16, d[c]);
        if (more) {
          ask(h[c], a.h, next * a.ldh, c, h_bf16);
          ask(dx[c], a.dx, next * a.lddx, c, dx_bf16);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) n[c][j] = inside(c, j) ? (n[c][j] - st.x) * st.y : 0.0f;
        if (mine && !COLS) {
          if (a.sum_out[0]) accumulate(Dw{}, c, d[c], n[c]);
          if constexpr (LAYER)
            if (a.sum_out[1]) accumulate(Dx{}, c, d[c], d[c]);
        }
        times(d[c], a.w, w[c], p_bf16);
      }
    }
    // Asked for while the row's sums are on their way.  Wide rows in turn: what the branch reads after the stream is stored.
    auto ask_branch = [&]() {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        if constexpr (!AHEAD) ask(g[c], a.gate, t * a.ldg, c, g_bf16);
        if constexpr (MODE == 2) {
          pw[c] = pb[c] = Piece{};
          ask(pw[c], a.pw, 0, c, p_bf16);
          if constexpr (LAYER)
            if (per_token) ask(pb[c], a.pb, 0, c, p_bf16);
        }
      }
    };
    constexpr bool kInTurn = !AHEAD && NCH > 1;
    if constexpr (kInTurn) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int c = 0; c < NCH; ++c) ask(dhi[c], a.dh_in, t * a.lddh_in, c, h_bf16);
    } else if constexpr (MODE >= 1) {
      ask_branch();
    }
    through(d, n, st.y);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      plus(d[c], a.dh_in, dhi[c], h_bf16);
      if (more) ask(dhi[c], a.dh_in, next * a.lddh_in, c, h_bf16);
      if (mine) piece_store<NT, VEC>(row_of(a.dh, t * a.lddh, h_bf16), c, lane, E, h_bf16, d[c]);
    }
    if constexpr (MODE >= 1) {
      if constexpr (kInTurn) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < NCH; ++c) ask(y[c], a.y, t * a.ldy, c, y_bf16);
        ask_branch();
      }
      // d: gradient of the stream.  n: y, or its normalised values
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        piece_values<VEC>(y[c], y_bf16, n[c]);
        if (more) ask(y[c], a.y, next * a.ldy, c, y_bf16);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (MODE == 2) n[c][j] = inside(c, j) ? (n[c][j] - st.z) * st.w : 0.0f;
          d[c][j] = inside(c, j) ? d[c][j] * a.scale : 0.0f;
        }
        if (per_token) {
          if (a.dgate) {
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = n[c][j];
            if constexpr (MODE == 2) {
              times(p, a.pw, pw[c], p_bf16);
              if constexpr (LAYER) plus(p, a.pb, pb[c], p_bf16);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] *= d[c][j];
            if (mine) piece_store<NT, VEC>(row_of(a.dgate, t * a.lddg, g_bf16), c, lane, E, g_bf16, p);
          }
          times(d[c], a.gate, g[c], g_bf16);
        }
        if (mine && !COLS) {
          if (want_qm) accumulate(Qm{}, c, d[c], n[c]);
          if constexpr (kSum[kQ])
            if (want_q) accumulate(Q{}, c, d[c], d[c]);
        }
        if (!per_token) times(d[c], a.gate, g[c], g_bf16);
        if (more) ask(g[c], a.gate, next * a.ldg, c, g_bf16);
        if constexpr (MODE == 2) times(d[c], a.pw, pw[c], p_bf16);
      }
      if constexpr (MODE == 2) through(d, n, st.w);
      if (a.dy && mine) {
#pragma unroll
        for (int c = 0; c < NCH; ++c) piece_store<NT, VEC>(row_of(a.dy, t * a.lddy, dy_bf16), c, lane, E, dy_bf16, d[c]);
      }
    }
  };
  if constexpr (LOOP) {
    for (int64_t first = (int64_t)blockIdx.x * TEAMS; first < a.T; first += step) rows(first);
  } else {
    rows((int64_t)(COLS ? blockIdx.x - a.column_groups : blockIdx.x) * TEAMS);
    if constexpr (COLS) return;
  }
  // ---- the workgroup's column sums, of its teams in order, and what they are the gradients of
  if constexpr (TEAMS > 1) {
    // Four columns to a lane of the first 2 NT (512 features, 4096 rows, against eight to the lanes of one team: 12.7 -> 11.2 us).
    // More than kBackwardRows rows: there is never a single workgroup here.
    static_assert(VEC && NCH == 1, "");
    __syncthreads();
    const int i = threadIdx.x, e = i * 4;
    if (i >= 2 * NT || e >= E) return;
    typedef float Four __attribute__((ext_vector_type(4)));
    Four total[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      total[s] = Four{0.0f, 0.0f, 0.0f, 0.0f};
      if (!kSum[s]) continue;
      const Four* q = reinterpret_cast<const Four*>(pool) + (kOrder[s] * 2 + i % 2) * (NT * TEAMS) + i / 2;
#pragma unroll
      for (int k = 0; k < TEAMS; ++k) total[s] = k == 0 ? q[0] : total[s] + q[k * NT];
    }
    auto four = [&](const void* p, int bf16) {
      if (bf16) {
        const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + e);
        return Four{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                    __uint_as_float(w.y & 0xFFFF0000u)};
      }
      return *reinterpret_cast<const Four*>(static_cast<const float*>(p) + e);
    };
    float* part = a.part;
    auto put = [&](float* to, Four v) {
      if (!to) return;
      *reinterpret_cast<Four*>(part + (int64_t)blockIdx.x * E + e) = v;
      part += (int64_t)gridDim.x * E;
    };
    put(a.sum_out[0], total[kDw]);
    if constexpr (LAYER) put(a.sum_out[1], total[kDx]);
    if constexpr (MODE >= 1) {
      if (a.sum_out[2]) {  // gate of one row: post_weight sum(q m) + post_bias sum(q)
        Four v = MODE == 2 && a.pw ? total[kQm] * four(a.pw, p_bf16) : total[kQm];
        if constexpr (kSum[kQ])
          if (a.pb) v += total[kQ] * four(a.pb, p_bf16);
        put(a.sum_out[2], v);
      }
      const bool one_row = a.gate && !per_token;
      const Four g1 = one_row ? four(a.gate, g_bf16) : Four{1.0f, 1.0f, 1.0f, 1.0f};
      put(a.sum_out[3], total[kQm] * g1);
      if constexpr (kSum[kQ]) put(a.sum_out[4], total[kQ] * g1);
    }
    return;
  }
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (!in_lds(s)) continue;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const float4 v = *slot(s, c, half, 0);
        const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[s][c][4 * half + j] = f[j];
      }
    }
    float* part = a.part;
    auto put = [&](float* to, const float (&v)[8]) {
      if (!to) return;
      if (gridDim.x == 1) {  // (a caller's array may lie anywhere)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (inside(c, j)) to[piece_at<NT, VEC>(c, j, lane)] = v[j];
        return;
      }
      piece_store<NT, VEC>(row_of(part, (int64_t)blockIdx.x * E, 0), c, lane, E, 0, v);
      part += (int64_t)gridDim.x * E;
    };
    put(a.sum_out[0], sum[kDw][c]);
    if constexpr (LAYER) put(a.sum_out[1], sum[kDx][c]);
    if constexpr (MODE >= 1) {
      Piece qg{}, qw{}, qb{};
      const bool one_row = a.gate && !per_token;
      if (one_row) ask(qg, a.gate, 0, c, g_bf16);
      if constexpr (MODE == 2) {
        ask(qw, a.pw, 0, c, p_bf16);
        if constexpr (LAYER) ask(qb, a.pb, 0, c, p_bf16);
      }
      float v[8];
      if (a.sum_out[2]) {  // gate of one row: post_weight sum(q m) + post_bias sum(q)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = sum[kQm][c][j];
        if constexpr (MODE == 2) times(v, a.pw, qw, p_bf16);
        if constexpr (kSum[kQ]) {
          float b[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) b[j] = sum[kQ][c][j];
          if (a.pb) {
            times(b, a.pb, qb, p_bf16);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += b[j];
          }
        }
        put(a.sum_out[2], v);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = sum[kQm][c][j];
      if (one_row) times(v, a.gate, qg, g_bf16);
      put(a.sum_out[3], v);
      if constexpr (kSum[kQ]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = sum[kQ][c][j];
        if (one_row) times(v, a.gate, qg, g_bf16);
        put(a.sum_out[4], v);
      }
    }
  }
}

}  // namespace blast_dev
