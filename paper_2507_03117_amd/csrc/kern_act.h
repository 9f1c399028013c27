// Gradient through an activation: dZ = dY act'(Z), gated dG = dH U act'(G), dU = dH act(G), H = act(G) U, with the column sums
// that are the biases' gradients (blast_act_backward in blast.h).
//
// Bound: memory, every operand read and every result written once.  A workgroup takes 256 columns, eight to a lane (16
// bytes of bf16), and a run of rows that its eight half-waves deal among themselves; the sums of a lane's columns stay in its
// registers over the run and meet in LDS at its end.
#pragma once
#include "kern_rows.h"

namespace blast_dev {

struct ActArgs {
  const void *z, *u, *dy;
  void *dz, *du, *h;
  float* part;         // [sum][run][N]; with one run the sums themselves
  float* sum_out[2];   // of dZ, of dU (null: not wanted)
  int64_t ldz, ldu, lddy, lddz, lddu, ldh;
  int T, N, run;       // run: rows of a workgroup
  int tiles;           // column tiles
  int dy_bf16, act;
};

// act(z) and act'(z)
__device__ __forceinline__ void act_and_slope(int act, float z, float& a, float& s) {
  if (act == BLAST_ACT_SILU) {
    const float g = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    a = z * g;
    s = g * __builtin_fmaf(z, 1.0f - g, 1.0f);
  } else if (act == BLAST_ACT_GELU) {
    // Phi(z) + z phi(z), Phi from the tail that gelu() has its values from
    const float t = __builtin_fabsf(z), tail = normal_tail(t);
    const float density = 0.39894228040143268f * __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
    s = __builtin_fmaf(z, density, z > 0.0f ? 1.0f - tail : tail);
    a = gelu(z);
  } else if (act == BLAST_ACT_RELU) {
    s = z > 0.0f ? 1.0f : 0.0f;
    a = z > 0.0f ? z : 0.0f;
  } else {
    s = 1.0f;
    a = z;
  }
}

constexpr int kActCols = 256, kActTeams = 8;

template <bool GATED, bool SUMS, bool VEC>
__global__ __launch_bounds__(256) void k_act_backward(const ActArgs a) {
  const int lane = threadIdx.x & 31, team = threadIdx.x >> 5;
  const int tile = (int)blockIdx.x % a.tiles, run = (int)blockIdx.x / a.tiles;
  const int col0 = tile * kActCols, width = a.N - col0 < kActCols ? a.N - col0 : kActCols;
  const int t_end = run * a.run + a.run < a.T ? run * a.run + a.run : a.T;
  float sum[2][8];
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[0][j] = sum[1][j] = 0.0f;
  for (int t = run * a.run + team; t < t_end; t += kActTeams) {
    Piece z{}, u{}, dy{};
    if (a.z) piece_load<32, VEC>(z, row_of(a.z, t * a.ldz + col0, 1), 0, lane, width, 1);
    if (GATED) piece_load<32, VEC>(u, row_of(a.u, t * a.ldu + col0, 1), 0, lane, width, 1);
    piece_load<32, VEC>(dy, row_of(a.dy, t * a.lddy + col0, a.dy_bf16), 0, lane, width, a.dy_bf16);
    float zv[8], uv[8], d[8], av[8], dz[8], du[8];
    piece_values<VEC>(z, 1, zv);
    piece_values<VEC>(dy, a.dy_bf16, d);
    if (GATED) piece_values<VEC>(u, 1, uv);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float slope;
      act_and_slope(a.act, zv[j], av[j], slope);
      dz[j] = GATED ? d[j] * uv[j] * slope : d[j] * slope;
      if (SUMS) sum[0][j] += dz[j];
      if (GATED) {
        du[j] = d[j] * av[j];
        av[j] *= uv[j];
        if (SUMS) sum[1][j] += du[j];
      }
    }
    if (a.dz) piece_store<32, VEC>(row_of(a.dz, t * a.lddz + col0, 1), 0, lane, width, 1, dz);
    if (GATED) {
      if (a.du) piece_store<32, VEC>(row_of(a.du, t * a.lddu + col0, 1), 0, lane, width, 1, du);
      if (a.h) piece_store<32, VEC>(row_of(a.h, t * a.ldh + col0, 1), 0, lane, width, 1, av);
    }
  }
  if constexpr (SUMS) {
    __shared__ float red[kActTeams][kActCols];
    const int runs = (a.T + a.run - 1) / a.run;
    float* out = a.part;
#pragma unroll
    for (int s = 0; s < (GATED ? 2 : 1); ++s) {
      if (!a.sum_out[s]) continue;
      float* dst = (runs == 1 ? a.sum_out[s] : out + (int64_t)run * a.N) + col0;
      out += (int64_t)runs * a.N;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) red[team][piece_at<32, VEC>(0, j, lane)] = sum[s][j];
      __syncthreads();
      const int e = threadIdx.x;
      if (e < width) {
        float v = red[0][e];
#pragma unroll
        for (int w = 1; w < kActTeams; ++w) v += red[w][e];
        dst[e] = v;
      }
    }
  }
}

}  // namespace blast_dev
