// Gradient of the stored blocks from activations kept in scaled 8-bit form: dvals[q] = sum over tokens of dY[t][row] X[t][col], the
// codes of X widened exactly to bf16 (a token has a scale of its own, which a sum over tokens cannot take outside).
//
// A workgroup of four waves has a stored block and a run of tokens.  A stage is 32 tokens for 128-wide blocks, 64 for 64-wide ones: dY as it
// is and X widened on the way into LDS, both turned by the transposing LDS read.  128-wide: a wave has a quadrant of the block;
// 64-wide: the whole of it for a quarter of the stage's tokens, and the four sums meet in LDS at the end.
#pragma once
#include "kern_scaled8.h"

namespace blast_dev {

struct Sddmm8Args {
  const int* row_ptr;
  const int* col_idx;
  const uint16_t* dy;
  int64_t ldy;
  Eight x;
  float* out;        // [run][nnz][b][b]
  int64_t out_run;   // elements between two runs' sums
  int T, nbr, nnz, runs, run_tokens;  // run_tokens: a multiple of a stage
};

template <int B>
struct Sd8Cfg {
  static constexpr int TOK = B == 128 ? 32 : 64;  // tokens of a stage
  static constexpr int ROWB = B * 2, TILE = TOK * ROWB, CPR = B / 8;
  static constexpr int LDS_BYTES = 2 * 2 * TILE;  // two stages; at the end four waves' sums, a quarter at a time
  __device__ static __forceinline__ int key(int row) { return 2 * (row & 3); }  // the four token rows of a transposing read on different banks
  __device__ static __forceinline__ uint32_t at(int row, int chunk) { return (uint32_t)(row * ROWB + ((chunk ^ key(row)) << 4)); }
};

template <int B>
__global__ __launch_bounds__(256) void k_sddmm8(const Sddmm8Args a) {
  using C = Sd8Cfg<B>;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[C::LDS_BYTES];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int q = blockIdx.x / a.runs, run = blockIdx.x % a.runs;
  int lo = 0, hi = a.nbr - 1;  // block row of q: the last r with row_ptr[r] <= q
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (ld_idx(a.row_ptr, mid) <= q) lo = mid; else hi = mid - 1;
  }
  const int64_t row0 = (int64_t)lo * B, col0 = (int64_t)ld_idx(a.col_idx, q) * B;
  const int t_lo = run * a.run_tokens, t_hi = t_lo + a.run_tokens < a.T ? t_lo + a.run_tokens : a.T;
  const int stages = (t_hi - t_lo + C::TOK - 1) / C::TOK;

  // what a thread copies of a stage: two 16-byte chunks of dY, sixteen codes of X and their token's scale
  const int yr[2] = {(int)threadIdx.x / C::CPR, ((int)threadIdx.x + 256) / C::CPR}, yc = threadIdx.x % C::CPR;
  const int xr = threadIdx.x / (B / 16), xc = threadIdx.x % (B / 16);
  const uint8_t* xscales = a.x.scales + ((col0 + xc * 16) >> a.x.shift) * a.x.lds;
  struct Stage {
    u32x4 y[2], x;
    int scale;
  };
  auto load = [&](int s) {
    Stage g;
    const int t0 = t_lo + s * C::TOK;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = t0 + yr[i];
      g.y[i] = u32x4{0, 0, 0, 0};
      if (t < a.T) g.y[i] = *reinterpret_cast<const u32x4*>(a.dy + t * a.ldy + row0 + yc * 8);
    }
    const int t = t0 + xr;
    g.x = u32x4{0, 0, 0, 0};
    g.scale = 127;
    if (t < a.T) {
      g.x = *reinterpret_cast<const u32x4*>(a.x.codes + t * a.x.ld + col0 + xc * 16);
      g.scale = xscales[t];
    }
    return g;
  };
  auto put = [&](const Stage& g, unsigned char* st) {
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<u32x4*>(st + C::at(yr[i], yc)) = g.y[i];
    const float scale = scale_value(g.scale);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x2v p = widen4(g.x[2 * i], a.x.fmt, scale), w = widen4(g.x[2 * i + 1], a.x.fmt, scale);
      *reinterpret_cast<u32x4*>(st + C::TILE + C::at(xr, 2 * xc + i)) = u32x4{p[0], p[1], w[0], w[1]};
    }
  };

  // Fragments: read h (0, 1) of a 32-wide tile takes token rows 8 (g / 2) + 4 h + p / 4 at features 16 (g % 2) + 4 (p % 4) of it, g the
  // lane's group of 16 and p its place there, and gives lane l the eight tokens 8 (l / 32) .. + 7 of feature l % 32.
  const int g16 = lane >> 4, p16 = lane & 15;
  const int wi = B == 128 ? wave >> 1 : 0, wj = B == 128 ? wave & 1 : 0;
  auto fragment = [&](const unsigned char* tile, int token0, int feature0) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    s16x4 h[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int row = token0 + 8 * (g16 >> 1) + 4 * k + (p16 >> 2), col = feature0 + 16 * (g16 & 1) + 4 * (p16 & 3);
      h[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4*)(tile + C::at(row, col >> 3) + (col & 7) * 2));
    }
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

  if (stages > 0) put(load(0), smem);
#pragma unroll 1
  for (int s = 0; s < stages; ++s) {
    Stage next;
    const bool more = s + 1 < stages;
    if (more) next = load(s + 1);
    __syncthreads();  // stage s is in LDS, and everybody has read s - 1
    const unsigned char* st = smem + (s & 1) * (2 * C::TILE);
#pragma unroll
    for (int k = 0; k < (B == 128 ? 2 : 1); ++k) {
      const int token0 = B == 128 ? 16 * k : 16 * wave;
      bf16x8 fy[2], fx[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fy[i] = fragment(st, token0, wi * 64 + 32 * i);
        fx[i] = fragment(st + C::TILE, token0, wj * 64 + 32 * i);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fy[i], fx[j], acc[i][j], 0, 0, 0);
    }
    if (more) put(next, smem + ((s + 1) & 1) * (2 * C::TILE));
  }

  float* out = a.out + run * a.out_run + (int64_t)q * (B * B);
  const int l32 = lane & 31, lh = lane >> 5;
  if constexpr (B == 128) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          __builtin_nontemporal_store(acc[i][j][v], out + (wi * 64 + 32 * i + 8 * (v >> 2) + 4 * lh + (v & 3)) * B + wj * 64 + 32 * j + l32);
  } else {
    // a tile of 32 x 32 at a time: the waves' four sums of it are added in wave order, four rows of registers to a wave
    float (*red)[16][64] = reinterpret_cast<float (*)[16][64]>(smem);
    static_assert(sizeof(float) * 4 * 16 * 64 <= C::LDS_BYTES, "");
#pragma unroll
    for (int tile = 0; tile < 4; ++tile) {
      const int i = tile >> 1, j = tile & 1;
      __syncthreads();
#pragma unroll
      for (int v = 0; v < 16; ++v) red[wave][v][lane] = acc[i][j][v];
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = wave * 4 + e;
        const float sum = ((red[0][v][lane] + red[1][v][lane]) + red[2][v][lane]) + red[3][v][lane];
        __builtin_nontemporal_store(sum, out + (32 * i + 8 * (v >> 2) + 4 * lh + (v & 3)) * B + 32 * j + l32);
      }
    }
  }
}

// The runs' sums of a block added in order.
static __global__ __launch_bounds__(256) void k_join_runs(const float* part, int64_t out_run, int runs, float* out, int64_t n) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= n) return;
  float4 s = *reinterpret_cast<const float4*>(part + i);
  for (int r = 1; r < runs; ++r) {
    const float4 p = *reinterpret_cast<const float4*>(part + r * out_run + i);
    s.x += p.x, s.y += p.y, s.z += p.z, s.w += p.w;
  }
  *reinterpret_cast<float4*>(out + i) = s;
}
static __global__ __launch_bounds__(256) void k_zero_blocks(float* out, int64_t n) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i < n) *reinterpret_cast<float4*>(out + i) = float4{0.0f, 0.0f, 0.0f, 0.0f};
}

}  // namespace blast_dev
