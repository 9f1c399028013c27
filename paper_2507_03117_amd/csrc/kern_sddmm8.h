// Gradient of the stored blocks from activations kept in scaled 8-bit form: dvals[q] = sum over tokens of dY[t][row] X[t][col], the
// codes of X widened exactly to bf16 (a token has a scale of its own, which a sum over tokens cannot take outside).
//
// k_sddmm8 (128-wide blocks): a workgroup of four waves has a block and a run of tokens, a wave a quadrant, so that a byte of the
// activations is read once a block.  A stage is 32 tokens: dY as it is and X widened on the way into LDS, both turned by the
// transposing LDS read.  Two stages are on their way in registers, the next is converted beside this one's matrix instructions.
// Bound: a stage's chain of LDS write, barrier, LDS read and matrix instructions, 0.5 us alone on a CU and 0.8 for two workgroups there, of
// which the matrix cores have 0.13 (179 blocks, 4096 tokens: 49 us with the joining of two runs, 6 of them, and 58 with inputs from memory;
// 75 before anything ran ahead, 66 with one stage ahead, 60 with conflicting LDS rows).  Its 358 workgroups of two runs leave 154 of 256
// CUs with one and 102 with two: stages dealt evenly would be 90 to a CU instead of up to 128.
//
// k_sddmm8_units (64-wide blocks; 128-wide ones where few have a middling number of tokens): a unit is a 64 x 64 part of a block and a
// run of tokens.  KW waves share it (four: they deal its stages of 16 tokens, and their sums meet in LDS in wave order; one: it has them
// all), UPW units make a workgroup.  There is no barrier before the sums: dY, the codes and their scales go by LDS-DMA into a ring of
// the wave's own.  A lane takes sixteen features of one token out of it, so that one scale serves it, and puts them back widened, a
// stage ahead of the one that is multiplied.  (Codes that come to registers cost a wait for everything in flight: the compiler
// does not count them apart from the copies.)
// Bound: the caches' rate for the activations, which each unit reads again (500 blocks of 64, 4096 tokens: 38 us, 50 with k_sddmm8's
// structure; 2867 blocks: 177 and 325; lane addresses that advance by scalars, fewer instructions, took as long or longer).
#pragma once
#include "kern_scaled8.h"
#include "kern_stream.h"

namespace blast_dev {

struct Sddmm8Args {
  const int* row_ptr;
  const int* col_idx;
  const uint16_t* dy;
  int64_t ldy;
  Eight x;
  float* out;        // [run][nnz][b][b]
  int64_t out_run;   // elements between two runs' sums
  int T, nbr, nnz, runs, run_tokens;  // run_tokens: a multiple of 64
  int n_units;  // of k_sddmm8_units: nnz (b / 64)^2 runs
};

struct Sd8Block {
  static constexpr int B = 128, TOK = 32;  // tokens of a stage
  static constexpr int ROWB = B * 2, TILE = TOK * ROWB, CPR = B / 8;
  static constexpr int LDS_BYTES = 2 * 2 * TILE;  // two stages
  // What half a wave's transposing read takes, four token rows of 64 bytes, lies on different banks of 64 (a row goes round them once).
  __device__ static __forceinline__ int key(int row) { return 4 * (row & 3); }
  __device__ static __forceinline__ uint32_t at(int row, int chunk) { return (uint32_t)(row * ROWB + ((chunk ^ key(row)) << 4)); }
};

constexpr int kAhead = 2;

template <int FMT>
__global__ __launch_bounds__(256) void k_sddmm8(const Sddmm8Args a) {
  using C = Sd8Block;
  constexpr int B = C::B;
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
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x2v p = widen4(g.x[2 * i], FMT, scale), w = widen4(g.x[2 * i + 1], FMT, scale);
      *reinterpret_cast<u32x4*>(st + C::TILE + C::at(xr, 2 * xc + i)) = u32x4{p[0], p[1], w[0], w[1]};
    }
  };

  // Fragments: read h (0, 1) of a 32-wide tile takes token rows 8 (g / 2) + 4 h + p / 4 at features 16 (g % 2) + 4 (p % 4) of it, g the
  // lane's group of 16 and p its place there, and gives lane l the eight tokens 8 (l / 32) .. + 7 of feature l % 32.
  const int g16 = lane >> 4, p16 = lane & 15;
  const int wi = wave >> 1, wj = wave & 1;
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
    for (int k = 0; k < 2; ++k) {
      bf16x8 fy[2], fx[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        fy[e] = fragment(st, 16 * k, wi * 64 + 32 * e);
        fx[e] = fragment(st + C::TILE, 16 * k, wj * 64 + 32 * e);
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
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        leave(acc[i][j][v], out + (wi * 64 + 32 * i + 8 * (v >> 2) + 4 * lh + (v & 3)) * B + wj * 64 + 32 * j + l32);
}

template <int B, int KW, int UPW>
struct Sd8Units {
  static constexpr int SUB = B / 64, KT = 16, AHEAD = 4;
  static constexpr int TILE = KT * 128;                    // 16 tokens of 64 bf16 values
  static constexpr int STAGE = TILE + KT * 64 + 256;       // dY, the codes, each lane's four scales
  static constexpr int OPS = 4;                            // copies of a stage
  static constexpr int WAVE_LDS = AHEAD * STAGE + 2 * TILE;  // the stages on their way, widened X of two
  static constexpr int NW = KW * UPW;
  static constexpr int LDS_BYTES = NW * WAVE_LDS;
  static_assert(KW == 1 || UPW == 1, "waves that share a unit meet at the workgroup's barrier");
  // The four token rows of a transposing read on different banks (rows of 128 bytes: two go round the 64 banks once).
  __device__ static __forceinline__ int key(int row) { return 4 * ((row >> 1) & 1); }
};

// The fragments of a stage: two 32-wide tiles of dY (addresses y0, y1) and of X (x0, x1), each in two halves of four token rows H bytes
// apart; and a lane's codes and scales of the next stage (addresses c, c4).  One block of assembly with its own wait: the compiler
// does not know the transposing read, and would wait for every copy before it reads what copies write.
template <int H>
__device__ __forceinline__ void sd8_read_stage(uint32_t y0, uint32_t y1, uint32_t x0, uint32_t x1, uint32_t c, uint32_t c4, u32x2v (&fr)[8],
                                               u32x4& code, uint32_t& scales) {
  asm volatile(
      "ds_read_b128 %8, %14\n\t"
      "ds_read_b32 %9, %15\n\t"
      "ds_read_b64_tr_b16 %0, %10 offset:0\n\t"
      "ds_read_b64_tr_b16 %1, %10 offset:%16\n\t"
      "ds_read_b64_tr_b16 %2, %11 offset:0\n\t"
      "ds_read_b64_tr_b16 %3, %11 offset:%16\n\t"
      "ds_read_b64_tr_b16 %4, %12 offset:0\n\t"
      "ds_read_b64_tr_b16 %5, %12 offset:%16\n\t"
      "ds_read_b64_tr_b16 %6, %13 offset:0\n\t"
      "ds_read_b64_tr_b16 %7, %13 offset:%16\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(fr[0]), "=&v"(fr[1]), "=&v"(fr[2]), "=&v"(fr[3]), "=&v"(fr[4]), "=&v"(fr[5]), "=&v"(fr[6]), "=&v"(fr[7]), "=&v"(code),
        "=&v"(scales)
      : "v"(y0), "v"(y1), "v"(x0), "v"(x1), "v"(c), "v"(c4), "n"(H)
      : "memory");
}
__device__ __forceinline__ void sd8_read_codes(uint32_t c, uint32_t c4, u32x4& code, uint32_t& scales) {
  asm volatile("ds_read_b128 %0, %2\n\tds_read_b32 %1, %3\n\ts_waitcnt lgkmcnt(0)" : "=&v"(code), "=&v"(scales) : "v"(c), "v"(c4) : "memory");
}

template <int B, int FMT, int KW, int UPW>
__global__ __launch_bounds__(64 * KW * UPW, 2) void k_sddmm8_units(const Sddmm8Args a) {
  using C = Sd8Units<B, KW, UPW>;
  constexpr int AHEAD = C::AHEAD;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wave = KW == 1 ? 0 : wv;  // place among the waves of the unit
  // ids go round the eight XCDs: neighbouring units, which read the same columns of dY or X, are eight apart, on one of them
  const int n_groups = (a.n_units + UPW - 1) / UPW, per_xcd = (n_groups + 7) >> 3;
  const int unit = (((int)blockIdx.x & 7) * per_xcd + ((int)blockIdx.x >> 3)) * UPW + (KW == 1 ? wv : 0);
  if (((int)blockIdx.x >> 3) >= per_xcd || unit >= a.n_units) return;  // every wave of a unit, before any barrier
  unsigned char* ring = smem + wv * C::WAVE_LDS;
  unsigned char* xbuf = ring + AHEAD * C::STAGE;

  const int run = unit % a.runs, rest = unit / a.runs;
  const int sj = rest % C::SUB, si = rest / C::SUB % C::SUB, q = rest / (C::SUB * C::SUB);
  int lo = 0, hi = a.nbr - 1;  // block row of q: the last r with row_ptr[r] <= q
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (ld_idx(a.row_ptr, mid) <= q) lo = mid; else hi = mid - 1;
  }
  const int64_t row0 = (int64_t)lo * B + si * 64, col0 = (int64_t)ld_idx(a.col_idx, q) * B + sj * 64;
  const int t_lo = run * a.run_tokens, t_hi = t_lo + a.run_tokens < a.T ? t_lo + a.run_tokens : a.T;
  const int all = t_hi > t_lo ? (t_hi - t_lo + C::KT - 1) / C::KT : 0;
  const int stages = all > wave ? (all - wave + KW - 1) / KW : 0;  // wave w has stages w, w + KW, ...

  // Copy side.  dY: instruction i writes bytes [i 1024 + lane 16, + 16) of a tile = token row 8 i + lane / 8, slot lane % 8, which holds
  // chunk slot ^ key(row) of it.  X: token lane / 4, features 16 (lane % 4) ... + 15.
  const int yrow = lane >> 3, xrow = lane >> 2, xc = lane & 3;
  const unsigned char* ybase = reinterpret_cast<const unsigned char*>(a.dy + row0);
  const uint8_t* xbase = a.x.codes + col0;
  const uint8_t* xscales = a.x.scales + (col0 >> a.x.shift) * a.x.lds;  // (64 features from a multiple of 64 on are of one group)
  const int last = a.T - 1;
  // Stages beyond the last ask for the last again, tokens beyond the last token for that one: what comes is not used, or made zeros.
  auto ask = [&](int s, int i) {
    const int st = s < stages ? s : stages - 1, t0 = t_lo + (wave + KW * st) * C::KT;
    unsigned char* stage = ring + i * C::STAGE;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int row = 8 * k + yrow, t = t0 + row < last ? t0 + row : last;
      BLAST_GLDS16(ybase + (int64_t)t * a.ldy * 2 + (((lane & 7) ^ C::key(row)) << 4), stage + k * 1024);
    }
    const int t = t0 + xrow < last ? t0 + xrow : last;
    BLAST_GLDS16(xbase + t * a.x.ld + xc * 16, stage + C::TILE);
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(xscales + (t & ~3)),
                                     (__attribute__((address_space(3))) void*)(stage + C::TILE + C::KT * 64), 4, 0, 0);
  };
  uint32_t xput[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) xput[k] = (uint32_t)(xrow * 128 + (((2 * xc + k) ^ C::key(xrow)) << 4));
  // (a stage begins at a multiple of 16: its tokens' places in their four are the lanes' own; those beyond the last token are made zeros)
  auto widen = [&](const u32x4& code, uint32_t scales, int half) {
    const float f = scale_value((scales >> (8 * (xrow & 3))) & 255);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const u32x2v p = widen4(code[2 * k], FMT, f), w = widen4(code[2 * k + 1], FMT, f);
      *reinterpret_cast<u32x4*>(xbuf + half * C::TILE + xput[k]) = u32x4{p[0], p[1], w[0], w[1]};
    }
  };

  // Fragment side: read h (0, 1) of a 32-wide tile takes token rows 8 (g / 2) + 4 h + p / 4 at features 16 (g % 2) + 4 (p % 4) of it, g
  // the lane's group of 16 and p its place there, and gives lane l the tokens 8 (l / 32) + 4 h ... + 3 of feature l % 32.
  const int g16 = lane >> 4, p16 = lane & 15;
  uint32_t foff[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int row = 8 * (g16 >> 1) + (p16 >> 2), col = 32 * n + 16 * (g16 & 1) + 4 * (p16 & 3);
    foff[n] = (uint32_t)(row * 128 + (((col >> 3) ^ C::key(row)) << 4) + (col & 7) * 2);
  }
  static_assert(C::AHEAD == 4, "key(row + 4) = key(row): the second half of a fragment lies 4 rows below the first");
  const uint32_t ring_addr = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)ring;
  const uint32_t x_addr = ring_addr + AHEAD * C::STAGE;
  const uint32_t codes = ring_addr + C::TILE + lane * 16, scales = ring_addr + C::TILE + C::KT * 64 + lane * 4;

  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
  auto multiply = [&](const u32x2v (&fr)[8]) {
    bf16x8 fy[2], fx[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      fy[n] = __builtin_bit_cast(bf16x8, (u32x4{fr[2 * n][0], fr[2 * n][1], fr[2 * n + 1][0], fr[2 * n + 1][1]}));
      fx[n] = __builtin_bit_cast(bf16x8, (u32x4{fr[4 + 2 * n][0], fr[4 + 2 * n][1], fr[5 + 2 * n][0], fr[5 + 2 * n][1]}));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fy[i], fx[j], acc[i][j], 0, 0, 0);
  };
  u32x4 code;
  uint32_t sc;
  // Stage i of the ring with the codes of the one behind it, of which nothing is still on its way: all but `pending` copies are there.
  auto read = [&](u32x2v (&fr)[8], int i) {
    const uint32_t y = ring_addr + i * C::STAGE, x = x_addr + (i & 1) * C::TILE, n = ((i + 1) & 3) * C::STAGE;
    __builtin_amdgcn_s_waitcnt(BLAST_VMCNT((AHEAD - 2) * C::OPS));
    asm volatile("" ::: "memory");
    sd8_read_stage<4 * 128>(y + foff[0], y + foff[1], x + foff[0], x + foff[1], codes + n, scales + n, fr, code, sc);
  };

  if (stages > 0) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ask(i, i);
    __builtin_amdgcn_s_waitcnt(BLAST_VMCNT((AHEAD - 1) * C::OPS));
    asm volatile("" ::: "memory");
    sd8_read_codes(codes, scales, code, sc);
    widen(code, sc, 0);
    int s0 = 0;
#pragma unroll 1
    for (; s0 + AHEAD < stages; s0 += AHEAD) {  // (never the last stage: the only one whose tokens may end in it)
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        u32x2v fr[8];
        read(fr, i);
        ask(s0 + i + AHEAD, i);
        widen(code, sc, (i + 1) & 1);
        multiply(fr);
      }
    }
    __builtin_amdgcn_s_waitcnt(BLAST_VMCNT(0));
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int s = s0 + i;
      if (s < stages) {
        u32x2v fr[8];
        read(fr, i);
        if (s + 1 < stages) widen(code, sc, (i + 1) & 1);
        const int valid = a.T - (t_lo + (wave + KW * s) * C::KT);
        if (valid < C::KT) {
          const int k0 = 8 * (lane >> 5);
#pragma unroll
          for (int f = 0; f < 8; ++f) {
            const int kf = k0 + 4 * (f & 1);  // the odd halves hold tokens k0 + 4 ... k0 + 7
#pragma unroll
            for (int w = 0; w < 2; ++w) {  // a register holds two tokens, the even one in its low half
              uint32_t v = fr[f][w];
              if (kf + 2 * w >= valid) v &= 0xFFFF0000u;
              if (kf + 2 * w + 1 >= valid) v &= 0x0000FFFFu;
              fr[f][w] = v;
            }
          }
        }
        multiply(fr);
      }
    }
  }

  float* out = a.out + run * a.out_run + (int64_t)q * (B * B) + (int64_t)(si * 64) * B + sj * 64;
  const int l32 = lane & 31, lh = lane >> 5;
  // (a sum that the next launch reads may stay in the caches)
  auto leave = [&](int i, int j, int v, float sum) {
    float* p = out + (32 * i + 8 * (v >> 2) + 4 * lh + (v & 3)) * B + 32 * j + l32;
    if (a.runs > 1)
      *p = sum;
    else
      __builtin_nontemporal_store(sum, p);
  };
  if constexpr (KW == 1) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) leave(i, j, v, acc[i][j][v]);
  } else {
    // two tiles of 32 x 32 at a time: the waves' four sums of them are added in wave order, eight rows of registers to a wave
    static_assert(KW == 4, "");
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
        const int e = wave * 8 + k;
        leave(i, e >> 4, e & 15, ((red[0][e][lane] + red[1][e][lane]) + red[2][e][lane]) + red[3][e][lane]);
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
