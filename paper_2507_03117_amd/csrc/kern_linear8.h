// Products of scaled 8-bit operands (kern_scaled8.h) over the stored blocks of a block row: one matrix with bias, activation and
// residual, or the gated pair; results in fp32, bf16 or scaled 8-bit form.  Features are the M dimension of the matrix instruction,
// tokens the N dimension: a lane has one token and hands over its scale with the codes.
//
// k_linear8: workgroups of four waves, two on a CU, walk lists of tiles: a block row's B rows of 128 tokens.  A step is 128 of the
// contraction: a stored block of 128 x 128 or two of 64 x 64, W and X tiles copied to LDS in rows of 128 bytes, the scales of the step's
// tokens beside them; the next step's copies are under way while one is multiplied, the next tile's first step while a tile's results leave
// (passes on the GPU alone: 53248 x 16384 at 95 %, 2048 tokens, a workgroup for each tile 199 us, lists 189; gated 14336 x 4096, 4096
// tokens, 106 / 100).
//
// Bound, 53248 x 16384 at 95 %, 2048 tokens, bf16: the widening, which every wave does for its own fragments, and the matrix instructions
// behind it: 37 and 43 % of the SIMDs' cycles by the counters, of which two waves a SIMD hide one behind the other only in part; beside
// that 0.66 GB read - a row's few blocks need other activations than the next row's, so that a byte of X is fetched for every block that
// reads it - and 0.22 written.  Gated 14336 x 4096 at 95 %, 4096 tokens, G, U and H kept in 8 bits, 97 to 100 us: 178 MB of results (20 us
// for G and U, 7 for SiLU) on top of the steps (60 us), which a row of 1.6 blocks a matrix keeps short; vector instructions take 44 % of
// the cycles, matrix instructions 19.  2048 x 8192 at 90 %, 64-wide, 2048 tokens, fp32 with an fp32 residual: 22 us, half of them bytes at
// a large copy's rate, the rest widened steps.
// Registers: 128 (one 64-wide matrix) to 248 (a 128-wide pair), no vector spills in any instance; 25 to 49 scalars of the tile kernel,
// addresses that results use, wait in lanes of a vector register.
// k_linear8_split: eight waves have a block row's B rows, or 32 of them, of 32 tokens and deal the stored blocks among themselves, W by way
// of LDS in whole lines, X straight into registers; their sums meet in LDS.  For calls whose 128-token tiles would leave CUs without work.
// Bound: a wave's chain of row, columns, blocks and X behind a launch (one token, 14336 x 4096 at 95 %, bf16 4.2 us, with whole rows 5.4;
// at 70 % 7.6 and 9.5, where widening counts; gated with 8-bit results 7.9 and 13.1; 64-wide 8192 x 2048 at 90 %, gated, five tokens 6.2;
// 1600 x 6400 at 80 %, 333 tokens 9.5; with bias and bf16 residual 9.7, 11 where they were asked for behind the sums).
#pragma once
#include "kern_scaled8.h"
#include "kern_stream.h"

namespace blast_dev {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct Mat8 {
  const int* row_ptr;
  const int* col_idx;
  const uint8_t* vals;
  const uint8_t* scales;
};

struct Linear8Args {
  Mat8 m[2];
  const int* row_order;  // may be null
  Eight x;
  int wfmt;
  int T, nbr, ntt;
  int parts;             // XCDs that share a block row, each with its own token tiles: 1 or 2
  int act;
  const float* bias;     // single matrix: all of these
  const void* r;
  int64_t ldr;
  int r_bf16;
  void* y;               // gated: H in bf16
  int64_t ldy;
  int y_bf16;
  int r_vec, y_vec;      // eight neighbouring rows of a token may be read / stored as one value
  Eight y8, k8[2];       // the result, what is kept (Z; G and U); codes null: not wanted
};

// Eight neighbouring rows of one token into a scaled 8-bit tensor; the lanes of a group are neighbours.
template <int B>
__device__ __forceinline__ void store_eight(const Eight& o, const float (&v)[8], int64_t t, int64_t row, bool live) {
  float w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = v[j];
  u32x2v codes;
  const int code = quantise8<B / 8>(w, o.fmt, codes);
  if (live) {
    *reinterpret_cast<u32x2v*>(o.codes + t * o.ld + row) = codes;
    if (row % B == 0) o.scales[(row / B) * o.lds + t] = (uint8_t)code;
  }
}

// Eight rows of a token of the residual, asked for.
__device__ __forceinline__ void ask_residual(const Linear8Args& a, Piece& q, int64_t t, int64_t row) {
  const unsigned char* p = row_of(a.r, t * a.ldr + row, a.r_bf16);
  if (a.r_vec)
    piece_load<1, true>(q, p, 0, 0, 8, a.r_bf16);
  else
    piece_load<1, false>(q, p, 0, 0, 8, a.r_bf16);
}

// Eight rows of a token from the sums to the outputs.  WHOLE: the workgroup has all B rows of it, which a scale is made of.
template <int B, bool DUAL, bool WHOLE>
__device__ __forceinline__ void linear8_finish(const Linear8Args& a, float (&z)[8], float (&u)[8], const float (&bias)[8],
                                               const Piece& residual, int64_t t, int64_t row, bool live) {
  if constexpr (DUAL) {
    if constexpr (WHOLE)
      if (a.k8[0].codes) store_eight<B>(a.k8[0], z, t, row, live);
    if constexpr (WHOLE)
      if (a.k8[1].codes) store_eight<B>(a.k8[1], u, t, row, live);
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = (a.act >= 0 ? epilogue_act(a.act, z[j]) : z[j]) * u[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] += bias[j];
    if constexpr (WHOLE)
      if (a.k8[0].codes) store_eight<B>(a.k8[0], z, t, row, live);
    if (a.act >= 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = epilogue_act(a.act, z[j]);
    }
    if (a.r && live) {
      float r[8];
      if (a.r_vec)
        piece_values<true>(residual, a.r_bf16, r);
      else
        piece_values<false>(residual, a.r_bf16, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] += r[j];
    }
  }
  if constexpr (WHOLE)
    if (a.y8.codes) store_eight<B>(a.y8, z, t, row, live);
  if (a.y && live) {
    unsigned char* p = row_of(a.y, t * a.ldy + row, a.y_bf16);
    if (a.y_vec)
      piece_store<1, true>(p, 0, 0, 8, a.y_bf16, z);
    else
      piece_store<1, false>(p, 0, 0, 8, a.y_bf16, z);
  }
}

// Codes widened to bf16 (exact), eight a 16-deep instruction.
__device__ __forceinline__ bf16x8 widen8(int lo, int hi, int fmt, float scale) {
  const u32x2v a = widen4((uint32_t)lo, fmt, scale), b = widen4((uint32_t)hi, fmt, scale);
  return __builtin_bit_cast(bf16x8, (u32x4{a[0], a[1], b[0], b[1]}));
}

// 64 of the contraction on 32 x 32 tiles: a lane has 32 bytes of a row of each operand, in formats WF and XF, the same places on both.  The
// 8-bit instructions take the codes as they are at two and a half times the rate, but hold a sum of 64 products in too few bits: they drop
// what lies 15 to 17 bits below the largest (448 and -448 beside 62 of 2^-9 give 0.10 for 0.12; 1.5e-5 root mean square of a sum of random
// terms, 4e-8 widened).  (The formats are constants: a branch at every conversion kept conversions and matrix instructions apart, 2048 x
// 8192 at 90 %, 2048 tokens, fp32 32.6 us, 21.2 without.)
template <int RT, int NT, int WF, int XF>
__device__ __forceinline__ void multiply8(f32x16 (&d)[RT][NT], const i32x8 (&fw)[RT], const i32x8 (&fx)[NT], int ws, const int (&xs)[NT]) {
  const float wsf = scale_value(ws);
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    bf16x8 bw[RT], bx[NT];
#pragma unroll
    for (int i = 0; i < RT; ++i) bw[i] = widen8(fw[i][2 * p], fw[i][2 * p + 1], WF, wsf);
#pragma unroll
    for (int j = 0; j < NT; ++j) bx[j] = widen8(fx[j][2 * p], fx[j][2 * p + 1], XF, scale_value(xs[j]));
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) d[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bw[i], bx[j], d[i][j], 0, 0, 0);
  }
}

// The tiles (block row, run of tokens) in eight lists, one for each XCD: an XCD has every (8 / parts)th block row and one of `parts`
// runs of the token tiles, a row's tiles one after the other.  Workgroup ids go round the XCDs; the workgroups of an XCD deal its list.
__device__ __forceinline__ bool place8(const Linear8Args& a, int item, int& rank, int& tt) {
  const int xcd = blockIdx.x & 7, per = (a.ntt + a.parts - 1) / a.parts, k = ((int)blockIdx.x >> 3) + item * ((int)gridDim.x >> 3);
  rank = k / per * (8 / a.parts) + xcd / a.parts;
  tt = xcd % a.parts * per + k % per;
  return rank < a.nbr && tt < a.ntt;
}
// How many of them this workgroup has.
__device__ __forceinline__ int items8(const Linear8Args& a) {
  const int xcd = blockIdx.x & 7, per = (a.ntt + a.parts - 1) / a.parts, rows = 8 / a.parts, mine = xcd / a.parts;
  const int n = (a.nbr > mine ? (a.nbr - mine + rows - 1) / rows : 0) * per, step = (int)gridDim.x >> 3, first = (int)blockIdx.x >> 3;
  return n > first ? (n - first + step - 1) / step : 0;
}

template <int B>
struct L8Cfg {
  static_assert(B == 64 || B == 128, "");
  static constexpr int NW = 4, TT = 32 * NW;  // tokens of a workgroup
  static constexpr int KB = 128 / B;            // stored blocks of a step
  static constexpr int WR = B / 64;             // waves along the rows, 64 each
  static constexpr int WT = NW / WR;            // waves along the tokens
  static constexpr int TW = TT / WT;            // tokens of a wave
  static constexpr int NT = TW / 32;
  static constexpr int W_BYTES = B * 128, X_BYTES = TT * 128;
  static constexpr int WI = W_BYTES / (1024 * NW), XI = X_BYTES / (1024 * NW);  // copy instructions of a wave, 1 KiB each
  static constexpr int S_BYTES = KB * 256;
  static constexpr int STAGE = W_BYTES + X_BYTES + S_BYTES;
  static constexpr int RING = 2 * STAGE;       // one step is multiplied, the next on its way
  static constexpr int EX_BYTES = 3 * WR * TT * 4;  // largest magnitudes that the waves of a token's rows tell each other
  static constexpr int LDS_BYTES = RING + EX_BYTES;
  static constexpr int OUT_BYTES = 4096;            // a wave's part of a stage when results leave
  static_assert(2 * B * TT <= STAGE && NW * OUT_BYTES <= STAGE && LDS_BYTES <= 160 * 1024, "");
};

// ---- results: a wave's 64 rows of 32 NT tokens, as the matrix instruction leaves them ----------------------------------------------
//
// Lane l has token l % 32 of a tile, register v row 8 (v / 4) + 4 (l / 32) + v % 4.  What leaves goes through a part of LDS that is the
// wave's own, [token][row], so that neighbouring lanes store neighbouring bytes: 16-byte chunk c of a token lies at c ^ key(token).

// f with the activation as a constant: decided once, not value by value.
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  if (act == BLAST_ACT_SILU)
    f(std::integral_constant<int, BLAST_ACT_SILU>{});
  else if (act == BLAST_ACT_GELU)
    f(std::integral_constant<int, BLAST_ACT_GELU>{});
  else if (act == BLAST_ACT_RELU)
    f(std::integral_constant<int, BLAST_ACT_RELU>{});
  else
    f(std::integral_constant<int, BLAST_ACT_NONE>{});
}
template <class A>
__device__ __forceinline__ float act_of(A, float z) {
  if constexpr (A::value == BLAST_ACT_NONE) return z;
  return epilogue_act(A::value, z);
}

// Bits of the largest magnitude of a token's values, over the two lanes that share it.  As integers the positive values are in their
// order and the negative ones, unsigned, above them in that of their magnitudes: two maxima and no sign taken off.  What is not finite
// (beyond kMostBits) is left out when it turns out to be there.
template <int NT>
__device__ __forceinline__ void token_max(const f32x16 (&d)[2][NT], uint32_t (&m)[NT]) {
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    int p = 0;
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int w = __float_as_int(d[i][j][v]);
        p = w > p ? w : p;
        n = (uint32_t)w > n ? (uint32_t)w : n;
      }
    n &= 0x7FFFFFFFu;
    uint32_t q = (uint32_t)p > n ? (uint32_t)p : n;
    if (__any(q >= 0x7F800000u)) {
      q = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const uint32_t u = magnitude(d[i][j][v]);
          if (u < 0x7F800000u) q = u > q ? u : q;
        }
    }
    const auto halves = __builtin_amdgcn_permlane32_swap(q, q, false, false);
    m[j] = halves[0] > halves[1] ? halves[0] : halves[1];
  }
}

// Codes of four values, a word.  CAP: finite magnitudes beyond kMostBits count as that.
template <int FMT, bool CAP>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float scale) {
  if constexpr (CAP) {
    auto cap = [](float x) {
      const uint32_t u = magnitude(x);
      return u > kMostBits && u < 0x7F800000u ? __builtin_copysignf(__uint_as_float(kMostBits), x) : x;
    };
    a = cap(a), b = cap(b), c = cap(c), d = cap(d);
  }
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  s16x2 w = {0, 0};
  if constexpr (FMT == BLAST_E4M3) {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
  } else {
    w = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(w, a, b, scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(w, c, d, scale, true);
  }
  return __builtin_bit_cast(uint32_t, w);
}

// A workgroup's codes of one tensor meet in LDS, [token][row], so that a token's B bytes - a whole line of 128 - leave together and past
// the L2s (bf16 results past the L2s too: 53248 x 16384 at 95 %, 2048 tokens 195 -> 189 us).
template <int B>
__device__ __forceinline__ uint32_t code_at(int tok, int chunk) {
  return (uint32_t)(tok * B + ((chunk ^ (B == 128 ? tok & 7 : (tok >> 1) & 3)) << 4));
}
template <int B, int NT, int FMT>
__device__ __forceinline__ void put_codes(const Eight& o, const f32x16 (&d)[2][NT], const uint32_t (&m)[NT], unsigned char* lds, int lane,
                                          int tok0, int row, int64_t t0, int64_t T, int group) {
  const int l32 = lane & 31, lh = lane >> 5;
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int tok = tok0 + 32 * j + l32;
    const int code = scale_code(m[j] > kMostBits ? kMostBits : m[j], FMT);
    const float scale = scale_value(code);
    if (row == 0 && lh == 0 && t0 + tok < T) o.scales[(int64_t)group * o.lds + t0 + tok] = (uint8_t)code;
    auto tile = [&](auto cap) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int v = 0; v < 16; v += 4)
          *reinterpret_cast<uint32_t*>(lds + code_at<B>(tok, (row >> 4) + 2 * i + (v >> 3)) + ((v & 4) ? 8 : 0) + 4 * lh) =
              encode4<FMT, decltype(cap)::value>(d[i][j][v], d[i][j][v + 1], d[i][j][v + 2], d[i][j][v + 3], scale);
    };
    if (__any(m[j] > kMostBits))
      tile(std::true_type{});
    else
      tile(std::false_type{});
  }
}
// This wave's 64 rows (from `row` on) of tokens tok0 ... of the workgroup's tile, whose first is t0.
template <int B, int NT>
__device__ __forceinline__ void put_eight(const Eight& o, const f32x16 (&d)[2][NT], const uint32_t (&m)[NT], unsigned char* lds, int lane,
                                          int tok0, int row, int64_t t0, int64_t T, int group) {
  if (o.fmt == BLAST_E4M3)
    put_codes<B, NT, BLAST_E4M3>(o, d, m, lds, lane, tok0, row, t0, T, group);
  else
    put_codes<B, NT, BLAST_E5M2>(o, d, m, lds, lane, tok0, row, t0, T, group);
}
// The tile's codes out of LDS, by all threads.
template <int B, int TT>
__device__ __forceinline__ void leave_eight(const Eight& o, const unsigned char* lds, int thread, int64_t t0, int64_t T, int64_t row0) {
  constexpr int kLanes = B / 16, kTokens = 256 / kLanes;
  const int c = thread % kLanes;
#pragma unroll
  for (int k = 0; k < TT / kTokens; ++k) {
    const int tok = k * kTokens + thread / kLanes;
    const u32x4 w = *reinterpret_cast<const u32x4*>(lds + code_at<B>(tok, c));
    if (t0 + tok < T) __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(o.codes + (t0 + tok) * o.ld + row0 + 16 * c));
  }
}

template <int NT>
__device__ __forceinline__ void put_bf16(uint16_t* y, int64_t ldy, bool vec, const f32x16 (&d)[2][NT], unsigned char* lds, int lane, int64_t t0,
                                         int64_t T, int64_t row0) {
  const int l32 = lane & 31, lh = lane >> 5, c = lane & 7;
#pragma unroll
  for (int j = 0; j < NT; ++j) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int v = 0; v < 16; v += 4)
        *reinterpret_cast<u32x2v*>(lds + l32 * 128 + (((4 * i + (v >> 2)) ^ (l32 & 7)) << 4) + 8 * lh) =
            u32x2v{bf16_pair(d[i][j][v], d[i][j][v + 1]), bf16_pair(d[i][j][v + 2], d[i][j][v + 3])};
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int tok = 8 * k + (lane >> 3);
      const int64_t t = t0 + 32 * j + tok;
      const u32x4 w = *reinterpret_cast<const u32x4*>(lds + tok * 128 + ((c ^ (tok & 7)) << 4));
      if (t < T) {
        uint16_t* p = y + t * ldy + row0 + 8 * c;
        if (vec) {
          __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p));
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Four neighbouring rows of a token's residual.
__device__ __forceinline__ void residual4(const Linear8Args& a, int64_t t, int64_t row, float (&r)[4]) {
  if (a.r_bf16) {
    const uint16_t* p = static_cast<const uint16_t*>(a.r) + t * a.ldr + row;
    uint32_t w[2];
    if (a.r_vec) {
      const u32x2v q = *reinterpret_cast<const u32x2v*>(p);
      w[0] = q[0], w[1] = q[1];
    } else {
      w[0] = p[0] | (uint32_t)p[1] << 16, w[1] = p[2] | (uint32_t)p[3] << 16;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = __uint_as_float(e % 2 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  } else {
    const float* p = static_cast<const float*>(a.r) + t * a.ldr + row;
    if (a.r_vec) {
      const float4 q = *reinterpret_cast<const float4*>(p);
      r[0] = q.x, r[1] = q.y, r[2] = q.z, r[3] = q.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = p[e];
    }
  }
}

// Values of either type with their residual, 16 tokens at a time: a lane takes four neighbouring rows of a token, a token's 64 are
// sixteen lanes'.
template <int NT>
__device__ __forceinline__ void put_sums(const Linear8Args& a, const f32x16 (&d)[2][NT], bool residual, unsigned char* lds, int lane,
                                         int64_t t0, int64_t row0) {
  const int l32 = lane & 31, lh = lane >> 5, c = lane & 15;
#pragma unroll
  for (int half = 0; half < 2 * NT; ++half) {
    const int j = half >> 1;
    const int64_t th = t0 + 16 * half;
    float r[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int e = 0; e < 4; ++e) r[k][e] = 0.0f;
      const int64_t t = th + 4 * k + (lane >> 4);
      if (residual && t < a.T) residual4(a, t, row0 + 4 * c, r[k]);
    }
    if ((l32 >> 4) == (half & 1)) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int v = 0; v < 16; v += 4)
          *reinterpret_cast<float4*>(lds + (l32 & 15) * 256 + (((8 * i + (v >> 1) + lh) ^ (l32 & 7)) << 4)) =
              float4{d[i][j][v], d[i][j][v + 1], d[i][j][v + 2], d[i][j][v + 3]};
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int tok = 4 * k + (lane >> 4);
      const int64_t t = th + tok;
      float4 w = *reinterpret_cast<const float4*>(lds + tok * 256 + ((c ^ (tok & 7)) << 4));
      w.x += r[k][0], w.y += r[k][1], w.z += r[k][2], w.w += r[k][3];
      if (t < a.T) {
        if (a.y_bf16) {
          uint16_t* p = static_cast<uint16_t*>(a.y) + t * a.ldy + row0 + 4 * c;
          if (a.y_vec) {
            *reinterpret_cast<u32x2v*>(p) = u32x2v{bf16_pair(w.x, w.y), bf16_pair(w.z, w.w)};
          } else {
            p[0] = f32_to_bf16_rne(w.x), p[1] = f32_to_bf16_rne(w.y), p[2] = f32_to_bf16_rne(w.z), p[3] = f32_to_bf16_rne(w.w);
          }
        } else {
          float* p = static_cast<float*>(a.y) + t * a.ldy + row0 + 4 * c;
          if (a.y_vec) {
            *reinterpret_cast<float4*>(p) = w;
          } else {
            p[0] = w.x, p[1] = w.y, p[2] = w.z, p[3] = w.w;
          }
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// What a workgroup has to do, one item a lane: block row, first token, first stored block and number of stored blocks of each matrix.
template <int NM, int TT>
struct Items8 {
  int row, t0, kb[NM], nb[NM];
  __device__ __forceinline__ void load(const Linear8Args& a, int first, int n, int lane) {
    row = t0 = 0;
#pragma unroll
    for (int m = 0; m < NM; ++m) kb[m] = nb[m] = 0;
    if (first + lane < n) {
      int rank, tt;
      const bool there = place8(a, first + lane, rank, tt);
      t0 = a.T;  // (a place beyond the last tile: no blocks, no token)
      if (there) {
        row = a.row_order ? a.row_order[rank] : rank;
        t0 = tt * TT;
#pragma unroll
        for (int m = 0; m < NM; ++m) {
          kb[m] = a.m[m].row_ptr[row];
          nb[m] = a.m[m].row_ptr[row + 1] - kb[m];
        }
      }
    }
  }
};

template <int B, bool DUAL, int WF, int XF>
__global__ __launch_bounds__(256, 2) void k_linear8(const Linear8Args a) {
  using C = L8Cfg<B>;
  constexpr int NW = C::NW, NT = C::NT, KB = C::KB, NM = DUAL ? 2 : 1, TT = C::TT;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l32 = lane & 31, lh = lane >> 5;
  const int wr = wave / C::WT, wt = wave % C::WT;  // this wave's 64 rows and TW tokens
  const int n_items = items8(a);
  if (n_items <= 0) return;

  // Copy side: position p (16 bytes) of a tile = row p / 8, slot p % 8; it holds chunk slot ^ row % 8 of that row's 128 bytes, which for
  // two blocks are 64 of each.  (row % 8 = lane / 8: a lane's chunk is the same in every instruction.)
  const int chunk = (lane & 7) ^ ((lane >> 3) & 7);
  const bool second = KB == 2 && chunk >= 4;  // it is of the second block
  const uint32_t coff = KB == 2 ? (chunk & 3) * 16 : chunk * 16;
  uint32_t woff[C::WI];
#pragma unroll
  for (int i = 0; i < C::WI; ++i) woff[i] = (uint32_t)(((i * NW + wave) * 8 + (lane >> 3)) * B) + coff;

  // The loader runs a step ahead of the multiplier, over the same sequence of items, matrices and steps.
  Items8<NM, TT> batch;
  int l_item = -1, l_m = NM - 1, l_s = 0, l_kb = 0, l_nb = 0, l_t0 = 0, l_c0 = 0, l_c1 = 0, l_slot = 0;
  bool l_valid = true;
  const uint8_t* xrow[C::XI];
  int64_t soff = 0;
  auto seek = [&]() {  // to the next step that there is
    while (l_s * KB >= l_nb) {
      l_s = 0;
      if (++l_m < NM) {
        l_kb = __builtin_amdgcn_readlane(batch.kb[NM - 1], l_item & 63);
        l_nb = __builtin_amdgcn_readlane(batch.nb[NM - 1], l_item & 63);
        continue;
      }
      l_m = 0;
      if (++l_item >= n_items) {
        l_valid = false;
        return;
      }
      if ((l_item & 63) == 0) batch.load(a, l_item, n_items, lane);
      l_kb = __builtin_amdgcn_readlane(batch.kb[0], l_item & 63);
      l_nb = __builtin_amdgcn_readlane(batch.nb[0], l_item & 63);
      l_t0 = __builtin_amdgcn_readlane(batch.t0, l_item & 63);
#pragma unroll
      for (int i = 0; i < C::XI; ++i) {
        int t = l_t0 + (i * NW + wave) * 8 + (lane >> 3);
        t = t < a.T ? t : a.T - 1;  // rows beyond the last token read it again; nothing of them is stored
        xrow[i] = a.x.codes + t * a.x.ld + coff;
      }
      soff = l_t0 + 4 * (lane < TT / 4 ? lane : TT / 4 - 1);
      soff = soff < a.x.lds - 4 ? soff : a.x.lds - 4;
    }
    const Mat8& m = a.m[DUAL ? l_m : 0];
    l_c0 = ld_idx(m.col_idx, l_kb + l_s * KB);
    l_c1 = KB == 2 && l_s * KB + 1 < l_nb ? ld_idx(m.col_idx, l_kb + l_s * KB + 1) : l_c0;
  };
  auto issue = [&]() {
    unsigned char* st = smem + l_slot * C::STAGE;
    const Mat8& m = a.m[DUAL ? l_m : 0];
    const int q0 = l_kb + l_s * KB, q1 = KB == 2 && l_s * KB + 1 < l_nb ? q0 + 1 : q0;
    const uint8_t* wsrc = m.vals + (int64_t)(second ? q1 : q0) * (B * B);
    const int64_t xcol = (int64_t)(second ? l_c1 : l_c0) * B;
#pragma unroll
    for (int i = 0; i < C::WI; ++i) BLAST_GLDS16(wsrc + woff[i], st + (i * NW + wave) * 1024);
#pragma unroll
    for (int i = 0; i < C::XI; ++i) BLAST_GLDS16(xrow[i] + xcol, st + C::W_BYTES + (i * NW + wave) * 1024);
    // (every wave copies the scales of one of the step's blocks: those that copy the same write the same)
    const int which = wave % KB, cs = which ? l_c1 : l_c0;
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void*)(a.x.scales + (((int64_t)cs * B) >> a.x.shift) * a.x.lds + soff),
        (__attribute__((address_space(3))) void*)(st + C::W_BYTES + C::X_BYTES + which * 256), 4, 0, 0);
    l_slot ^= 1;
    ++l_s;
    seek();
  };

  f32x16 acc[NM][2][NT];
  // Fragment side: of each 64 of a row lane half h takes chunks h and h + 2, the same on both operands.
  auto chunk_at = [&](int row, int c) { return (uint32_t)(row * 128 + ((c ^ (row & 7)) << 4)); };
  auto multiply = [&](f32x16 (&d)[2][NT], int w0, int w1, bool two, int slot) {
    const unsigned char* st = smem + slot * C::STAGE;
    const unsigned char* sc = st + C::W_BYTES + C::X_BYTES;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      if (KB == 2 && kk == 1 && !two) break;  // (an odd number of blocks)
      i32x8 fw[2], fx[NT];
      int xs[NT];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = wr * 64 + 32 * i + l32;
        const i32x4 lo = *reinterpret_cast<const i32x4*>(st + chunk_at(row, 4 * kk + lh));
        const i32x4 hi = *reinterpret_cast<const i32x4*>(st + chunk_at(row, 4 * kk + lh + 2));
        fw[i] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int row = wt * C::TW + 32 * j + l32;
        const i32x4 lo = *reinterpret_cast<const i32x4*>(st + C::W_BYTES + chunk_at(row, 4 * kk + lh));
        const i32x4 hi = *reinterpret_cast<const i32x4*>(st + C::W_BYTES + chunk_at(row, 4 * kk + lh + 2));
        fx[j] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        xs[j] = sc[(KB == 2 ? kk : 0) * 256 + row];
      }
      multiply8<2, NT, WF, XF>(d, fw, fx, kk && KB == 2 ? w1 : w0, xs);
    }
  };

  int slot = 0;  // of the step multiplied next
  auto meet = [&]() {  // all waves' LDS accesses so far; no copy is waited for
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto run = [&](f32x16 (&d)[2][NT], const Mat8& m, int kb, int nb) {
#pragma unroll 1
    for (int b0 = 0; b0 < nb; b0 += KB) {
      const int q = kb + b0;
      const bool two = KB == 2 && b0 + 1 < nb;
      const int w0 = (ld_idx(reinterpret_cast<const int*>(m.scales), q >> 2) >> (8 * (q & 3))) & 255;
      const int w1 = two ? (ld_idx(reinterpret_cast<const int*>(m.scales), (q + 1) >> 2) >> (8 * ((q + 1) & 3))) & 255 : w0;
      __builtin_amdgcn_s_waitcnt(BLAST_VMCNT(0));  // this step's copies: no others are under way
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): what was read of the step before is here
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();  // everybody's copies of this step have landed, and the stage of the step before is free
      asm volatile("" ::: "memory");
      if (l_valid) issue();
      multiply(d, w0, w1, two, slot);
      slot ^= 1;
    }
  };

  seek();
  if (l_valid) issue();

  Items8<NM, TT> mine;
#pragma unroll 1
  for (int item = 0; item < n_items; ++item) {
    if ((item & 63) == 0) mine.load(a, item, n_items, lane);
    const int r = __builtin_amdgcn_readlane(mine.row, item & 63), t0 = __builtin_amdgcn_readlane(mine.t0, item & 63);
#pragma unroll
    for (int m = 0; m < NM; ++m) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[m][i][j][v] = 0.0f;
      run(acc[m], a.m[m], __builtin_amdgcn_readlane(mine.kb[m], item & 63), __builtin_amdgcn_readlane(mine.nb[m], item & 63));
    }

    // Results, by way of the stage that no copy is on its way to.  `ex`: largest magnitudes over a wave's rows of each token, of up to
    // three tensors; a group of 128 rows is two waves'.
    int ln = lane;
    asm volatile("" : "+v"(ln));  // (what follows from it is made here again, not kept in registers through the steps)
    const int l32 = ln & 31, lh = ln >> 5, thread = wave * 64 + ln;
    unsigned char* stage = smem + (slot ^ 1) * C::STAGE;
    unsigned char* lds = stage + wave * C::OUT_BYTES;
    uint32_t* ex = reinterpret_cast<uint32_t*>(smem + C::RING);
    const int64_t tw = t0 + wt * C::TW, row0 = (int64_t)r * B + wr * 64;
    auto tell = [&](int k, const uint32_t (&m)[NT]) {
      if (lh == 0) {
#pragma unroll
        for (int j = 0; j < NT; ++j) ex[(k * C::WR + wr) * TT + wt * C::TW + 32 * j + l32] = m[j];
      }
    };
    auto told = [&](int k, uint32_t (&m)[NT]) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        m[j] = 0;
#pragma unroll
        for (int w = 0; w < C::WR; ++w) {
          const uint32_t o = ex[(k * C::WR + w) * TT + wt * C::TW + 32 * j + l32];
          m[j] = o > m[j] ? o : m[j];
        }
      }
    };
    constexpr int kCodes = B * TT;  // bytes of the tile's codes
    const int tok0 = wt * C::TW;
    const int64_t rows0 = (int64_t)r * B;
    if constexpr (DUAL) {
      const bool keep_g = a.k8[0].codes, keep_u = a.k8[1].codes, to8 = a.y8.codes;
      uint32_t m[NT];
      if (keep_g) token_max<NT>(acc[0], m), tell(0, m);
      if (keep_u) token_max<NT>(acc[1], m), tell(1, m);
      meet();  // (everybody has read the last step; what was told can be heard)
      if (keep_g) told(0, m), put_eight<B, NT>(a.k8[0], acc[0], m, stage, ln, tok0, wr * 64, t0, a.T, r);
      if (keep_u) told(1, m), put_eight<B, NT>(a.k8[1], acc[1], m, stage + kCodes, ln, tok0, wr * 64, t0, a.T, r);
      f32x16 (&h)[2][NT] = acc[0];
      with_act(a.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) h[i][j][v] = act_of(act, h[i][j][v]) * acc[1][i][j][v];
      });
      if (to8) token_max<NT>(h, m), tell(2, m);
      meet();  // (G's and U's codes are in LDS)
      if (keep_g) leave_eight<B, TT>(a.k8[0], stage, thread, t0, a.T, rows0);
      if (keep_u) leave_eight<B, TT>(a.k8[1], stage + kCodes, thread, t0, a.T, rows0);
      meet();  // (and out of it)
      if (to8) {
        told(2, m), put_eight<B, NT>(a.y8, h, m, stage, ln, tok0, wr * 64, t0, a.T, r);
        meet();
        leave_eight<B, TT>(a.y8, stage, thread, t0, a.T, rows0);
      } else {
        put_bf16<NT>(static_cast<uint16_t*>(a.y), a.ldy, a.y_vec, h, lds, ln, tw, a.T, row0);
      }
    } else {
      f32x16 (&d)[2][NT] = acc[0];
      if (a.bias) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const float b = a.bias[row0 + 32 * i + 8 * (v >> 2) + 4 * lh + (v & 3)];
#pragma unroll
            for (int j = 0; j < NT; ++j) d[i][j][v] += b;
          }
      }
      const bool keep = a.k8[0].codes, to8 = a.y8.codes;
      uint32_t m[NT];
      if (keep) token_max<NT>(d, m), tell(0, m);
      meet();  // (everybody has read the last step; what was told can be heard)
      if (keep) {
        told(0, m), put_eight<B, NT>(a.k8[0], d, m, stage, ln, tok0, wr * 64, t0, a.T, r);
        meet();
        leave_eight<B, TT>(a.k8[0], stage, thread, t0, a.T, rows0);
        meet();
      }
      with_act(a.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) d[i][j][v] = act_of(act, d[i][j][v]);
      });
      const bool added = to8 && a.r;  // (before the result is written: it may be where the residual is)
      if (added) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int64_t t = tw + 32 * j + l32;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; v += 4) {
              float q[4] = {0.0f, 0.0f, 0.0f, 0.0f};
              if (t < a.T) residual4(a, t, row0 + 32 * i + 2 * v + 4 * lh, q);
#pragma unroll
              for (int e = 0; e < 4; ++e) d[i][j][v + e] += q[e];
            }
        }
      }
      if (a.y) {
        if (!a.y_bf16 || (a.r && !added))
          put_sums<NT>(a, d, a.r && !added, lds, ln, tw, row0);
        else
          put_bf16<NT>(static_cast<uint16_t*>(a.y), a.ldy, a.y_vec, d, lds, ln, tw, a.T, row0);
      }
      if (to8) {
        token_max<NT>(d, m), tell(1, m);
        meet();
        told(1, m), put_eight<B, NT>(a.y8, d, m, stage, ln, tok0, wr * 64, t0, a.T, r);
        meet();
        leave_eight<B, TT>(a.y8, stage, thread, t0, a.T, rows0);
      }
    }
  }
}

// ---- few tiles: waves share the stored blocks of a block row ------------------------------------------------------------------

template <int B, int ROWS, bool DUAL>
struct S8Cfg {
  static constexpr int NW = 8, TT = 32, RT = ROWS / 32;
  static constexpr int EP_TOKENS = DUAL && ROWS == 128 ? 16 : 32;  // tokens whose sums lie in LDS at once, of every wave and matrix
  static constexpr int W_BYTES = ROWS * B;  // a wave's block
  static constexpr int SUM_BYTES = NW * EP_TOKENS * ROWS * 4 * (DUAL ? 2 : 1), LDS_BYTES = SUM_BYTES > NW * W_BYTES ? SUM_BYTES : NW * W_BYTES;
  // 16-byte chunk c of a row lies at c ^ key(row): eight rows' chunks of a fragment are on different banks.
  __device__ static __forceinline__ int key(int row) { return B == 128 ? row & 7 : (row >> 1) & 3; }
};

// ROWS: of a block row's B, the workgroup's (blockIdx.y says which).  The sums are the same in either form.
template <int B, int ROWS, bool DUAL, int WF, int XF>
__global__ __launch_bounds__(512) void k_linear8_split(const Linear8Args a) {
  using C = S8Cfg<B, ROWS, DUAL>;
  constexpr int NM = DUAL ? 2 : 1, RT = C::RT, NW = C::NW, KS = B / 64;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l32 = lane & 31, lh = lane >> 5;
  int rank, tt;
  if (!place8(a, 0, rank, tt)) return;
  const int r = a.row_order ? ld_idx(a.row_order, rank) : rank;
  const int t0 = tt * C::TT;
  int kb[NM], nb[NM];
#pragma unroll
  for (int m = 0; m < NM; ++m) {
    kb[m] = ld_idx(a.m[m].row_ptr, r);
    nb[m] = ld_idx(a.m[m].row_ptr, r + 1) - kb[m];
  }
  const int64_t t = t0 + l32 < a.T ? t0 + l32 : a.T - 1;  // (lanes beyond the last token repeat it; nothing of them is stored)
  const uint8_t* xrow = a.x.codes + t * a.x.ld + lh * 32;

  constexpr int kPieces = ROWS / 8, kRows = 64 * NW / kPieces, PITCH = ROWS * 4, SET = C::EP_TOKENS * PITCH;
  const int piece = threadIdx.x % kPieces;
  const int64_t row = (int64_t)r * B + (int)blockIdx.y * ROWS + piece * 8;
  // what a thread adds to its sums (of one token, if there is anything to add), on its way from the start
  float bias[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  Piece residual{};
  if constexpr (!DUAL) {
    static_assert(kRows >= C::EP_TOKENS && C::EP_TOKENS == C::TT, "");
    if (a.bias) {
#pragma unroll
      for (int j = 0; j < 8; ++j) bias[j] = a.bias[row + j];
    }
    const int64_t tk = t0 + (int)threadIdx.x / kPieces;
    if (a.r && (int)threadIdx.x / kPieces < C::TT && tk < a.T) ask_residual(a, residual, tk, row);
  }
  f32x16 acc[NM][RT][1];
#pragma unroll
  for (int m = 0; m < NM; ++m)
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[m][i][0][v] = 0.0f;

  // W by way of LDS, a block to a wave's own part of it: whole lines are asked for, where a fragment's 32 bytes a row would ask for each
  // line again and again.  The next block is on its way beside the matrix instructions.
  unsigned char* mine = smem + wave * C::W_BYTES;
  struct Ahead {
    i32x8 x[KS];
    int xs, ws;
  };
  auto ask = [&](Ahead& n, const Mat8& m, int q) {
    constexpr int kSlots = B / 16;
    const uint8_t* w = m.vals + (int64_t)q * (B * B) + (int)blockIdx.y * ROWS * B;
#pragma unroll
    for (int i = 0; i < C::W_BYTES / 1024; ++i) {
      const int row = i * (64 / kSlots) + lane / kSlots;
      BLAST_GLDS16(w + row * B + (((lane % kSlots) ^ C::key(row)) << 4), mine + i * 1024);
    }
    const int c = ld_idx(m.col_idx, q);
    n.ws = (ld_idx(reinterpret_cast<const int*>(m.scales), q >> 2) >> (8 * (q & 3))) & 255;
    n.xs = a.x.scales[(((int64_t)c * B) >> a.x.shift) * a.x.lds + t];
    const uint8_t* x = xrow + (int64_t)c * B;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const i32x4* p = reinterpret_cast<const i32x4*>(x + k * 64);
      n.x[k] = __builtin_shufflevector(p[0], p[1], 0, 1, 2, 3, 4, 5, 6, 7);
    }
  };
  auto blocks = [&](f32x16 (&d)[RT][1], const Mat8& m, int first, int q0, int n) {
    if (first >= n) return;
    Ahead next;
    ask(next, m, q0 + first);
#pragma unroll 1
    for (int e = first; e < n; e += NW) {
      const Ahead now = next;
      const int xs[1] = {now.xs};
      __builtin_amdgcn_s_waitcnt(BLAST_VMCNT(0));
      asm volatile("" ::: "memory");
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        i32x8 fw[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          const int row = i * 32 + l32;
          i32x4 h[2];
#pragma unroll
          for (int p = 0; p < 2; ++p)
            h[p] = *reinterpret_cast<const i32x4*>(mine + row * B + (((k * 4 + lh * 2 + p) ^ C::key(row)) << 4));
          fw[i] = __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
        }
        if (k == KS - 1 && e + NW < n) {
          __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the part is read before it is written again
          asm volatile("" ::: "memory");
          ask(next, m, q0 + e + NW);
        }
        const i32x8 fx[1] = {now.x[k]};
        multiply8<RT, 1, WF, XF>(d, fw, fx, now.ws, xs);
      }
    }
  };
  // the blocks of both matrices are dealt as one sequence
  blocks(acc[0], a.m[0], wave, kb[0], nb[0]);
  if constexpr (DUAL) blocks(acc[1], a.m[1], (wave + NW - nb[0] % NW) % NW, kb[1], nb[1]);

  const int all = nb[0] + (DUAL ? nb[NM - 1] : 0), waves = all < NW ? (all < 1 ? 1 : all) : NW;  // those that have sums
#pragma unroll 1
  for (int pass = 0; pass < C::TT / C::EP_TOKENS; ++pass) {
    if (t0 + pass * C::EP_TOKENS >= a.T) break;
    __syncthreads();
    const int tok = l32 - pass * C::EP_TOKENS;
    if (wave < waves && tok >= 0 && tok < C::EP_TOKENS && t0 + l32 < a.T) {
#pragma unroll
      for (int m = 0; m < NM; ++m) {
        unsigned char* base = smem + (wave * NM + m) * SET + tok * PITCH;
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int v = 0; v < 16; v += 4) {
            const int c = (32 * i + 2 * v + 4 * lh) / 4;
            *reinterpret_cast<float4*>(base + ((c ^ (tok & 7)) << 4)) =
                float4{acc[m][i][0][v], acc[m][i][0][v + 1], acc[m][i][0][v + 2], acc[m][i][0][v + 3]};
          }
      }
    }
    __syncthreads();
#pragma unroll 1
    for (int k = threadIdx.x / kPieces; k < C::EP_TOKENS; k += kRows) {
      const int64_t tk = t0 + pass * C::EP_TOKENS + k;
      if (t0 + pass * C::EP_TOKENS + (k & ~(kRows - 1)) >= a.T) break;
      float z[8], u[8];
      auto take = [&](int m, float (&v)[8]) {  // the waves' sums in their order
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
#pragma unroll 1
        for (int w0 = 0; w0 < waves; w0 += 2) {  // two at a time: their reads are under way together
          float4 lo[2], hi[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const unsigned char* base = smem + ((w0 + i) * NM + m) * SET + k * PITCH;
            lo[i] = *reinterpret_cast<const float4*>(base + (((2 * piece) ^ (k & 7)) << 4));
            hi[i] = *reinterpret_cast<const float4*>(base + (((2 * piece + 1) ^ (k & 7)) << 4));
          }
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (i == 0 || w0 + i < waves)
              v[0] += lo[i].x, v[1] += lo[i].y, v[2] += lo[i].z, v[3] += lo[i].w, v[4] += hi[i].x, v[5] += hi[i].y, v[6] += hi[i].z,
                  v[7] += hi[i].w;
        }
      };
      take(0, z);
      if constexpr (DUAL) take(1, u);
      linear8_finish<B, DUAL, ROWS == B>(a, z, u, bias, residual, tk, row, tk < a.T);
    }
  }
}

}  // namespace blast_dev
