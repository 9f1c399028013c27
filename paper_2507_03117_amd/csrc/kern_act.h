// Gradient through an activation: dZ = dY act'(Z), gated dG = dH U act'(G), dU = dH act(G), H = act(G) U, with the column sums
// that are the biases' gradients (blast_act_backward in blast.h).
//
// Bound: memory, every operand read and every result written once.  A workgroup takes 256 columns, eight to a lane (16
// bytes of bf16), and a run of rows that its eight half-waves deal among themselves; the sums of a lane's columns stay in its
// registers over the run and meet in LDS at its end, those of the runs in a second launch - or, for few rows, a workgroup has its
// columns' rows to the end (k_act_backward_columns).  Measured: gated, 4096 x 14336, fp32 gradient 163 us (5.05 TB/s, the rate of a
// large copy); GELU with the bias' gradient, 333 x 6400 7.4 us, 4096 x 6400 39 us.
#pragma once
#include "kern_rows.h"

namespace blast_dev {

struct ActArgs {
  const void *z, *u, *dy;
  void *dz, *du, *h;
  float* part;         // [sum wanted][run][N] (a single run writes sum_out instead)
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
    a = z <= 0.0f ? 0.0f : z;  // (a NaN stays one)
  } else {
    s = 1.0f;
    a = z;
  }
}

// One row of a lane's eight columns: what is read of it, and what is made of that; the sums over the rows that a lane has
// had in `sum`.  NL lanes share a row.
struct ActRow {
  Piece z, u, dy;
};
template <int NL, bool GATED, bool VEC>
__device__ __forceinline__ void act_read(const ActArgs& a, ActRow& q, int t, int col0, int lane, int width) {
  q = ActRow{};
  if (a.z) piece_load<NL, VEC>(q.z, row_of(a.z, t * a.ldz + col0, 1), 0, lane, width, 1);
  if (GATED) piece_load<NL, VEC>(q.u, row_of(a.u, t * a.ldu + col0, 1), 0, lane, width, 1);
  piece_load<NL, VEC>(q.dy, row_of(a.dy, t * a.lddy + col0, a.dy_bf16), 0, lane, width, a.dy_bf16);
}
template <int NL, bool GATED, bool SUMS, bool VEC>
__device__ __forceinline__ void act_write(const ActArgs& a, const ActRow& q, int t, int col0, int lane, int width, float (&sum)[2][8]) {
  float zv[8], uv[8], d[8], av[8], dz[8], du[8];
  piece_values<VEC>(q.z, 1, zv);
  piece_values<VEC>(q.dy, a.dy_bf16, d);
  if (GATED) piece_values<VEC>(q.u, 1, uv);
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
  if (a.dz) piece_store<NL, VEC>(row_of(a.dz, t * a.lddz + col0, 1), 0, lane, width, 1, dz);
  if (GATED) {
    if (a.du) piece_store<NL, VEC>(row_of(a.du, t * a.lddu + col0, 1), 0, lane, width, 1, du);
    if (a.h) piece_store<NL, VEC>(row_of(a.h, t * a.ldh + col0, 1), 0, lane, width, 1, av);
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
    ActRow q;
    act_read<32, GATED, VEC>(a, q, t, col0, lane, width);
    act_write<32, GATED, SUMS, VEC>(a, q, t, col0, lane, width, sum);
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

// The same with the sums in one launch: a workgroup has 32 columns of all rows, four lanes to a row, two rows of a lane on
// their way at a time, and nothing is left to be joined afterwards.  Two neighbouring workgroups of an XCD (ids eight apart)
// share the 128-byte lines of bf16.
constexpr int kActOwned = 32;
template <bool GATED, bool VEC, int THREADS>
__global__ __launch_bounds__(THREADS) void k_act_backward_columns(const ActArgs a) {
  constexpr int kLanes = kActOwned / 8, kRows = THREADS / kLanes, kWaves = THREADS / 64;
  const int lane = threadIdx.x % kLanes, team = threadIdx.x / kLanes, id = blockIdx.x;
  const int col0 = ((id / 16) * 16 + (id % 8) * 2 + id / 8 % 2) * kActOwned;
  const int width = a.N - col0 < kActOwned ? a.N - col0 : kActOwned;
  if (width <= 0) return;
  float sum[2][8];
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[0][j] = sum[1][j] = 0.0f;
  for (int t = team; t < a.T; t += 2 * kRows) {
    ActRow q0, q1;
    act_read<kLanes, GATED, VEC>(a, q0, t, col0, lane, width);
    const bool two = t + kRows < a.T;
    if (two) act_read<kLanes, GATED, VEC>(a, q1, t + kRows, col0, lane, width);
    act_write<kLanes, GATED, true, VEC>(a, q0, t, col0, lane, width, sum);
    if (two) act_write<kLanes, GATED, true, VEC>(a, q1, t + kRows, col0, lane, width, sum);
  }
  // the sixteen rows of a wave, then the waves in order
  __shared__ float red[kWaves][kActOwned];
#pragma unroll
  for (int s = 0; s < (GATED ? 2 : 1); ++s) {
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

}  // namespace blast_dev
