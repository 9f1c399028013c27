// Products of scaled 8-bit operands (kern_scaled8.h) over the stored blocks of a block row: one matrix with bias, activation and
// residual, or the gated pair; results in fp32, bf16 or scaled 8-bit form.
//
// A workgroup of four waves has a block row's B rows of TT tokens.  A step is 128 of the contraction: a stored block of 128 x 128
// or two of 64 x 64, W and X tiles copied to LDS in rows of 128 bytes, the scales of the step's tokens beside them.  Features are the M
// dimension of the matrix instruction, tokens the N dimension: a lane has one token and hands over its scale with the codes.
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

// Eight rows of a token from the sums to the outputs.
template <int B, bool DUAL>
__device__ __forceinline__ void linear8_finish(const Linear8Args& a, float (&z)[8], float (&u)[8], const float (&bias)[8], int64_t t,
                                               int64_t row, bool live) {
  if constexpr (DUAL) {
    if (a.k8[0].codes) store_eight<B>(a.k8[0], z, t, row, live);
    if (a.k8[1].codes) store_eight<B>(a.k8[1], u, t, row, live);
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = (a.act >= 0 ? epilogue_act(a.act, z[j]) : z[j]) * u[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] += bias[j];
    if (a.k8[0].codes) store_eight<B>(a.k8[0], z, t, row, live);
    if (a.act >= 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = epilogue_act(a.act, z[j]);
    }
    if (a.r && live) {
      Piece q{};
      float r[8];
      const unsigned char* p = row_of(a.r, t * a.ldr + row, a.r_bf16);
      if (a.r_vec) {
        piece_load<1, true>(q, p, 0, 0, 8, a.r_bf16);
        piece_values<true>(q, a.r_bf16, r);
      } else {
        piece_load<1, false>(q, p, 0, 0, 8, a.r_bf16);
        piece_values<false>(q, a.r_bf16, r);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] += r[j];
    }
  }
  if (a.y8.codes) store_eight<B>(a.y8, z, t, row, live);
  if (a.y && live) {
    unsigned char* p = row_of(a.y, t * a.ldy + row, a.y_bf16);
    if (a.y_vec)
      piece_store<1, true>(p, 0, 0, 8, a.y_bf16, z);
    else
      piece_store<1, false>(p, 0, 0, 8, a.y_bf16, z);
  }
}

// One step of the contraction on 32 x 32 tiles: sixteen bytes twice of each operand's row are a lane's share of 64.
template <int WF, int XF>
__device__ __forceinline__ f32x16 mfma8(i32x8 w, i32x8 x, f32x16 c, int ws, int xs) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, c, WF, XF, 0, ws, 0, xs);
}
// The same codes widened to bf16, eight a 16-deep instruction.
__device__ __forceinline__ bf16x8 widen8(int lo, int hi, int fmt, float scale) {
  const u32x2v a = widen4((uint32_t)lo, fmt, scale), b = widen4((uint32_t)hi, fmt, scale);
  return __builtin_bit_cast(bf16x8, (u32x4{a[0], a[1], b[0], b[1]}));
}

template <int B, int TT, bool DUAL>
struct L8Cfg {
  static_assert(B == 64 || B == 128, "");
  static constexpr int KB = 128 / B;            // stored blocks of a step
  static constexpr int WR = B / 64;             // waves along the rows, 64 each
  static constexpr int WT = 4 / WR;             // waves along the tokens
  static constexpr int TW = TT / WT;            // tokens of a wave
  static constexpr int NT = TW / 32;
  static constexpr int W_BYTES = B * 128, X_BYTES = TT * 128;
  static constexpr int WI = W_BYTES / 4096, XI = X_BYTES / 4096;  // copy instructions of a wave, 1 KiB each
  static constexpr int S_BYTES = 4 * 256;       // scales of the step's tokens: a wave copies those of one of its blocks
  static constexpr int STAGE = W_BYTES + X_BYTES + S_BYTES;
  static constexpr int NSTAGE = 2;
  static constexpr int EP_TOKENS = DUAL || TT * B * 4 > NSTAGE * STAGE ? TT / 2 : TT;  // tokens whose sums lie in LDS at once
  static constexpr int EP_BYTES = EP_TOKENS * B * 4 * (DUAL ? 2 : 1);
  static constexpr int LDS_BYTES = NSTAGE * STAGE > EP_BYTES ? NSTAGE * STAGE : EP_BYTES;
};

template <int B, int TT, bool DUAL, bool EXACT>
__global__ __launch_bounds__(256) void k_linear8(const Linear8Args a) {
  using C = L8Cfg<B, TT, DUAL>;
  constexpr int NT = C::NT, KB = C::KB, NM = DUAL ? 2 : 1;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l32 = lane & 31, lh = lane >> 5;
  // ids go round the eight XCDs: the token tiles of a block row are eight apart, on one of them
  const int id = blockIdx.x, span = 8 * a.ntt, rem = id % span;
  const int rank = id / span * 8 + (rem & 7), tt = rem >> 3;
  if (rank >= a.nbr) return;
  const int r = a.row_order ? ld_idx(a.row_order, rank) : rank;
  const int t0 = tt * TT;
  const int wr = wave / C::WT, wt = wave % C::WT;  // this wave's 64 rows and TW tokens

  int kb[NM], nb[NM], steps[NM];
#pragma unroll
  for (int m = 0; m < NM; ++m) {
    kb[m] = ld_idx(a.m[m].row_ptr, r);
    nb[m] = ld_idx(a.m[m].row_ptr, r + 1) - kb[m];
    steps[m] = (nb[m] + KB - 1) / KB;
  }
  const int total = steps[0] + (DUAL ? steps[NM - 1] : 0);

  // Copy side: position p (16 bytes) of a tile = row p / 8, slot p % 8; it holds chunk slot ^ row % 8 of that row's 128 bytes, which for
  // two blocks are 64 of each.
  uint32_t woff[C::WI];
  const uint8_t* xrow[C::XI];
#pragma unroll
  for (int i = 0; i < C::WI; ++i) {
    const int p = (i * 4 + wave) * 64 + lane, row = p >> 3, c = (p & 7) ^ (row & 7);
    woff[i] = (uint32_t)(KB == 2 ? row * 64 + (c & 3) * 16 : row * 128 + c * 16);
  }
#pragma unroll
  for (int i = 0; i < C::XI; ++i) {
    const int p = (i * 4 + wave) * 64 + lane, row = p >> 3, c = (p & 7) ^ (row & 7);
    int t = t0 + row;
    t = t < a.T ? t : a.T - 1;  // rows beyond the last token read it again; nothing of them is stored
    xrow[i] = a.x.codes + t * a.x.ld + (KB == 2 ? (c & 3) * 16 : c * 16);
  }
  int64_t soff = t0 + 4 * (lane < TT / 4 ? lane : TT / 4 - 1);
  soff = soff < a.x.lds - 4 ? soff : a.x.lds - 4;
  const bool second = KB == 2 && (((lane & 7) ^ ((lane >> 3) & 7)) >= 4);  // (row % 8 = lane / 8: this lane's chunk is of the second block)

  auto issue = [&](int m, int s, int slot) {
    unsigned char* st = smem + slot * C::STAGE;
    const int q0 = kb[m] + s * KB;
    const int q1 = KB == 2 && s * KB + 1 < nb[m] ? q0 + 1 : q0;
    const int c0 = ld_idx(a.m[m].col_idx, q0), c1 = KB == 2 ? ld_idx(a.m[m].col_idx, q1) : c0;
    const uint8_t* wsrc = a.m[m].vals + (int64_t)(second ? q1 : q0) * (B * B);
    const int64_t xcol = (int64_t)(second ? c1 : c0) * B;
#pragma unroll
    for (int i = 0; i < C::WI; ++i) BLAST_GLDS16(wsrc + woff[i], st + (i * 4 + wave) * 1024);
#pragma unroll
    for (int i = 0; i < C::XI; ++i) BLAST_GLDS16(xrow[i] + xcol, st + C::W_BYTES + (i * 4 + wave) * 1024);
    const int cs = KB == 2 && (wave & 1) ? c1 : c0;
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void*)(a.x.scales + (((int64_t)cs * B) >> a.x.shift) * a.x.lds + soff),
        (__attribute__((address_space(3))) void*)(st + C::W_BYTES + C::X_BYTES + wave * 256), 4, 0, 0);
  };

  f32x16 acc[NM][2][NT];
#pragma unroll
  for (int m = 0; m < NM; ++m)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[m][i][j][v] = 0.0f;

  // Fragment side: of each 64 of a row lane half h takes chunks h and h + 2, the same on both operands.
  auto chunk_at = [&](int row, int c) { return (uint32_t)(row * 128 + ((c ^ (row & 7)) << 4)); };
  auto multiply = [&](f32x16 (&d)[2][NT], int m, int s, int slot) {
    const unsigned char* st = smem + slot * C::STAGE;
    const unsigned char* sc = st + C::W_BYTES + C::X_BYTES;
    const int q0 = kb[m] + s * KB;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      if (KB == 2 && kk == 1 && s * KB + 1 >= nb[m]) break;  // (an odd number of blocks)
      const int q = q0 + (KB == 2 ? kk : 0);
      const int ws = (ld_idx(reinterpret_cast<const int*>(a.m[m].scales), q >> 2) >> (8 * (q & 3))) & 255;  // (through the scalar unit)
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
      if constexpr (EXACT) {
        const float wsf = scale_value(ws);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          bf16x8 bw[2], bx[NT];
#pragma unroll
          for (int i = 0; i < 2; ++i) bw[i] = widen8(fw[i][2 * p], fw[i][2 * p + 1], a.wfmt, wsf);
#pragma unroll
          for (int j = 0; j < NT; ++j) bx[j] = widen8(fx[j][2 * p], fx[j][2 * p + 1], a.x.fmt, scale_value(xs[j]));
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) d[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bw[i], bx[j], d[i][j], 0, 0, 0);
        }
      } else {
        auto all = [&](auto wf, auto xf) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) d[i][j] = mfma8<wf.value, xf.value>(fw[i], fx[j], d[i][j], ws, xs[j]);
        };
        using F0 = std::integral_constant<int, 0>;
        using F1 = std::integral_constant<int, 1>;
        if (a.wfmt == BLAST_E4M3) {
          if (a.x.fmt == BLAST_E4M3)
            all(F0{}, F0{});
          else
            all(F0{}, F1{});
        } else {
          if (a.x.fmt == BLAST_E4M3)
            all(F1{}, F0{});
          else
            all(F1{}, F1{});
        }
      }
    }
  };

  auto issue_step = [&](int g, int slot) {
    if (!DUAL || g < steps[0])
      issue(0, g, slot);
    else
      issue(NM - 1, g - steps[0], slot);
  };
  if (total > 0) issue_step(0, 0);
#pragma unroll 1
  for (int g = 0; g < total; ++g) {
    __syncthreads();  // (waits for this wave's copies: step g's have landed, everybody has read step g - 1)
    if (g + 1 < total) issue_step(g + 1, (g + 1) & 1);
    if (!DUAL || g < steps[0])
      multiply(acc[0], 0, g, g & 1);
    else
      multiply(acc[NM - 1], NM - 1, g - steps[0], g & 1);
  }

  // The sums through LDS, [token][row] in fp32, so that a lane ends with eight neighbouring rows of a token: 16-byte chunk c of a token
  // lies at c ^ token % 8.
  constexpr int kPieces = B / 8, kRows = 256 / kPieces, PITCH = B * 4;
  const int piece = threadIdx.x % kPieces;
  const int64_t row = (int64_t)r * B + piece * 8;
  float bias[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) bias[j] = !DUAL && a.bias ? a.bias[row + j] : 0.0f;
#pragma unroll
  for (int pass = 0; pass < TT / C::EP_TOKENS; ++pass) {
    __syncthreads();
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int tok = wt * C::TW + 32 * j + l32 - pass * C::EP_TOKENS;
        if (tok >= 0 && tok < C::EP_TOKENS) {
          unsigned char* base = smem + m * (C::EP_TOKENS * PITCH) + tok * PITCH;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; v += 4) {
              const int c = (wr * 64 + 32 * i + 2 * v + 4 * lh) / 4;
              *reinterpret_cast<float4*>(base + ((c ^ (tok & 7)) << 4)) =
                  float4{acc[m][i][j][v], acc[m][i][j][v + 1], acc[m][i][j][v + 2], acc[m][i][j][v + 3]};
            }
        }
      }
    __syncthreads();
#pragma unroll 1
    for (int tok = threadIdx.x / kPieces; tok < C::EP_TOKENS; tok += kRows) {
      const int64_t t = t0 + pass * C::EP_TOKENS + tok;
      if (t0 + pass * C::EP_TOKENS + (tok & ~(kRows - 1)) >= a.T) break;  // (the same for the workgroup)
      float z[8], u[8];
      auto take = [&](int m, float (&v)[8]) {
        const unsigned char* base = smem + m * (C::EP_TOKENS * PITCH) + tok * PITCH;
        const float4 lo = *reinterpret_cast<const float4*>(base + (((2 * piece) ^ (tok & 7)) << 4));
        const float4 hi = *reinterpret_cast<const float4*>(base + (((2 * piece + 1) ^ (tok & 7)) << 4));
        v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
      };
      take(0, z);
      if constexpr (DUAL) take(1, u);
      linear8_finish<B, DUAL>(a, z, u, bias, t, row, t < a.T);
    }
  }
}

}  // namespace blast_dev
