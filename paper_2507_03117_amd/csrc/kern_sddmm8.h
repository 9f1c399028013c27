// Gradient of the stored blocks from activations kept in scaled 8-bit form: dvals[q] = sum over tokens of dY[t][row] X[t][col], the
// codes of X widened exactly to bf16 (a token has a scale of its own, which a sum over tokens cannot take outside).
//
// A workgroup of four waves has a stored block and a run of tokens.  A stage is 32 tokens for 128-wide blocks, 64 for 64-wide ones: dY as it
// is and X widened on the way into LDS, both turned by the transposing LDS read.  128-wide: a wave has a quadrant of the block, so
// that a byte of the activations is read once a block; 64-wide: the whole of it for a quarter of the stage's tokens, and the four sums
// meet in LDS at the end.  Two stages are on their way in registers, the next is converted beside this one's matrix instructions.
//
// Bound: a stage's chain of LDS write, barrier, LDS read and matrix instructions, 0.5 us alone on a CU and 0.8 for two workgroups there, of
// which the matrix cores have 0.13 (179 blocks of 128 x 128, 4096 tokens: 59 us with the joining of two runs, 6 of them; 75 before
// anything ran ahead, 66 with one stage ahead, 60 with conflicting LDS rows).
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
  // What half a wave's transposing read takes, four token rows of 64 bytes, lies on different banks of 64 (two rows of 128 bytes, or one
  // of 256, go round them once).
  __device__ static __forceinline__ int key(int row) { return B == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1); }
  __device__ static __forceinline__ uint32_t at(int row, int chunk) { return (uint32_t)(row * ROWB + ((chunk ^ key(row)) << 4)); }
};

constexpr int kAhead = 2;

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
  // Tokens beyond the last read it again, and are made zeros on the way into LDS: no load depends on a comparison.
  auto load = [&](Stage& g, int s) {
    const int t0 = t_lo + s * C::TOK;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = t0 + yr[i] < a.T ? t0 + yr[i] : a.T - 1;
      g.y[i] = *reinterpret_cast<const u32x4*>(a.dy + t * a.ldy + row0 + yc * 8);
    }
    const int t = t0 + xr < a.T ? t0 + xr : a.T - 1;
    g.x = *reinterpret_cast<const u32x4*>(a.x.codes + t * a.x.ld + col0 + xc * 16);
    g.scale = xscales[t];
  };
  auto put = [&](Stage& g, unsigned char* st, int s) {
    const int t0 = t_lo + s * C::TOK;
    if (t0 + C::TOK > a.T) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (t0 + yr[i] >= a.T) g.y[i] = u32x4{0, 0, 0, 0};
      if (t0 + xr >= a.T) g.x = u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<u32x4*>(st + C::at(yr[i], yc)) = g.y[i];
    const float scale = scale_value(g.scale);
    auto widen = [&](auto fmt) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const u32x2v p = widen4(g.x[2 * i], fmt.value, scale), w = widen4(g.x[2 * i + 1], fmt.value, scale);
        *reinterpret_cast<u32x4*>(st + C::TILE + C::at(xr, 2 * xc + i)) = u32x4{p[0], p[1], w[0], w[1]};
      }
    };
    if (a.x.fmt == BLAST_E4M3)
      widen(std::integral_constant<int, BLAST_E4M3>{});
    else
      widen(std::integral_constant<int, BLAST_E5M2>{});
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

  // kAhead stages are on their way to registers while one is multiplied.  The next one goes into the other half of LDS beside the matrix
  // instructions: that half was read before the barrier that lets this one be read.
  Stage next[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) load(next[k], k < stages ? k : stages - 1);
  auto multiply = [&](const unsigned char* st) {
#pragma unroll
    for (int k = 0; k < (B == 128 ? 2 : 1); ++k) {
      const int token0 = B == 128 ? 16 * k : 16 * wave;
      bf16x8 fy[2], fx[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        fy[e] = fragment(st, token0, wi * 64 + 32 * e);
        fx[e] = fragment(st + C::TILE, token0, wj * 64 + 32 * e);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int f = 0; f < 2; ++f) acc[e][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fy[e], fx[f], acc[e][f], 0, 0, 0);
    }
  };
  auto meet = [&]() {
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0); what is on its way to registers need not be waited for
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  put(next[0], smem, 0);
  load(next[0], kAhead < stages ? kAhead : stages - 1);
  int s0 = 0;
#pragma unroll 1
  for (; s0 + kAhead < stages; s0 += kAhead) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int s = s0 + i, half = (s & 1) * (2 * C::TILE);
      meet();
      multiply(smem + half);
      Stage& g = next[(i + 1) % kAhead];
      put(g, smem + (2 * C::TILE - half), s + 1);
      load(g, s + 1 + kAhead < stages ? s + 1 + kAhead : stages - 1);
    }
  }
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const int s = s0 + i, half = (s & 1) * (2 * C::TILE);
    if (s < stages) {
      meet();
      multiply(smem + half);
      if (s + 1 < stages) put(next[(i + 1) % kAhead], smem + (2 * C::TILE - half), s + 1);
    }
  }

  float* out = a.out + run * a.out_run + (int64_t)q * (B * B);
  const int l32 = lane & 31, lh = lane >> 5;
  // (a sum that the next launch reads may stay in the caches)
  auto leave = [&](float v, float* p) {
    if (a.runs > 1)
      *p = v;
    else
      __builtin_nontemporal_store(v, p);
  };
  if constexpr (B == 128) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          leave(acc[i][j][v], out + (wi * 64 + 32 * i + 8 * (v >> 2) + 4 * lh + (v & 3)) * B + wj * 64 + 32 * j + l32);
  } else {
    // two tiles of 32 x 32 at a time: the waves' four sums of them are added in wave order, eight rows of registers to a wave
    float (*red)[32][64] = reinterpret_cast<float (*)[32][64]>(smem);
    static_assert(sizeof(float) * 4 * 32 * 64 <= C::LDS_BYTES, "");
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 32; ++e) red[wave][e][lane] = acc[i][e >> 4][e & 15];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int e = wave * 8 + k, j = e >> 4, v = e & 15;
        const float sum = ((red[0][e][lane] + red[1][e][lane]) + red[2][e][lane]) + red[3][e][lane];
        leave(sum, out + (32 * i + 8 * (v >> 2) + 4 * lh + (v & 3)) * B + 32 * j + l32);
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
