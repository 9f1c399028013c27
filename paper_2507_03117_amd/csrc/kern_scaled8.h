// Scaled 8-bit tensors: codes in E4M3 or E5M2 with a power of two for each token and group of 64 or 128 features (blast_scaled8_view
// in blast.h), and the conversions to and from them.
//
// The scale of a group is 2^e, e the smallest integer from -100 on with amax <= 1.75 * 2^(P + e), 1.75 * 2^P the format's largest value
// (448, 57344): division by it is exact, a code depends on its value and its group's exponent alone, every value a code stands for is
// a bf16 value (so that the gradient of the stored blocks loses nothing when it widens them), and the matrix instructions of the
// f8f6f4 family take the exponents as they are stored.  Below 2^-100 a scale would bring code values under the smallest normal bf16.
//
// Bound: memory, every value read and every code written once; a lane has sixteen bytes or more of a row, a group's lanes find its maximum
// by lane exchanges, a wave has four tokens so that their scales leave as one word (4096 x 14336, bf16: 33 us, 5.3 TB/s, a large copy's rate;
// one token of 2048: 2.6, a launch).
#pragma once
#include "kern_rows.h"

namespace blast_dev {

typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
typedef float f32x2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

struct Eight {
  uint8_t* codes;
  uint8_t* scales;  // [groups][lds]
  int64_t ld, lds;
  int fmt;          // BLAST_E4M3 / BLAST_E5M2
  int shift;        // log2 of the group
};

constexpr int kLeastScale = 127 - 100;
constexpr uint32_t kMostBits = 0x7F600000u;  // 1.75 * 2^127: a finite magnitude beyond it counts as that (rounded up it would be 2^128)

// Biased exponent of a group's scale from the bits of its largest magnitude.
__device__ __forceinline__ int scale_code(uint32_t amax, int fmt) {
  const int e = (int)(amax >> 23) + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0) - (fmt == BLAST_E4M3 ? 8 : 15);
  return e > kLeastScale ? e : kLeastScale;
}
__device__ __forceinline__ float scale_value(int code) { return __uint_as_float((uint32_t)code << 23); }
__device__ __forceinline__ float scale_inverse(int code) { return __uint_as_float((uint32_t)(254 - code) << 23); }

// Largest of a value over the LANES (8 or 16) neighbouring lanes of a group, in all of them.
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t m) {
  auto step = [&](auto ctrl) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, ctrl.value, 0xF, 0xF, true);
    m = o > m ? o : m;
  };
  step(std::integral_constant<int, 0xB1>{});   // quads: lanes 1 0 3 2
  step(std::integral_constant<int, 0x4E>{});   // 2 3 0 1
  step(std::integral_constant<int, 0x141>{});  // half rows turned round
  if constexpr (LANES == 16) step(std::integral_constant<int, 0x140>{});  // rows turned round
  return m;
}

// Eight codes of eight values, already divided by their scale.
__device__ __forceinline__ u32x2v encode8(const float (&v)[8], int fmt) {
  u32x2v w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int c = 0;
    if (fmt == BLAST_E4M3) {
      c = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], c, false);
      c = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], c, true);
    } else {
      c = __builtin_amdgcn_cvt_pk_bf8_f32(v[4 * i], v[4 * i + 1], c, false);
      c = __builtin_amdgcn_cvt_pk_bf8_f32(v[4 * i + 2], v[4 * i + 3], c, true);
    }
    w[i] = (uint32_t)c;
  }
  return w;
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// The values of a group's lanes to codes: returns the group's scale.  NaN and infinity (E4M3 has none: NaN) keep out of the scale.
template <int LANES>
__device__ __forceinline__ int quantise8(float (&v)[8], int fmt, u32x2v& codes) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t a = magnitude(v[j]);
    m = a > m ? a : m;
  }
  m = lanes_max<LANES>(m);
  if (m > kMostBits) {  // (rare) something is not finite, or too large to be rounded up
    m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t a = magnitude(v[j]);
      if (a < 0x7F800000u) {
        if (a > kMostBits) {
          a = kMostBits;
          v[j] = __builtin_copysignf(__uint_as_float(kMostBits), v[j]);
        }
        m = a > m ? a : m;
      }
    }
    m = lanes_max<LANES>(m);
  }
  const int code = scale_code(m, fmt);
  const float inv = scale_inverse(code);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= inv;
  codes = encode8(v, fmt);
  return code;
}

// What eight codes stand for.
__device__ __forceinline__ void decode8(u32x2v w, int fmt, float scale, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    f32x2v lo, hi;
    if (fmt == BLAST_E4M3) {
      lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], scale, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], scale, true);
    } else {
      lo = __builtin_amdgcn_cvt_scalef32_pk_f32_bf8(w[i], scale, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_f32_bf8(w[i], scale, true);
    }
    v[4 * i] = lo[0];
    v[4 * i + 1] = lo[1];
    v[4 * i + 2] = hi[0];
    v[4 * i + 3] = hi[1];
  }
}
__device__ __forceinline__ float decode1(uint8_t c, int fmt, float scale) {
  return fmt == BLAST_E4M3 ? __builtin_amdgcn_cvt_scalef32_f32_fp8(c, scale, 0) : __builtin_amdgcn_cvt_scalef32_f32_bf8(c, scale, 0);
}
// Four codes as bf16 values (exact).
__device__ __forceinline__ u32x2v widen4(uint32_t w, int fmt, float scale) {
  bf16x2v lo, hi;
  if (fmt == BLAST_E4M3) {
    lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
  } else {
    lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, true);
  }
  return u32x2v{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// ---- an activation into that form and back -------------------------------------------------------------------------------

struct KeepArgs {
  Eight q;
  const void* x;  // the other side: read by the quantiser, written by the other
  int64_t ldx;
  int64_t T, K;
  int x_bf16;
  int tiles;      // of 512 columns
};

// A wave has 512 columns, eight to a lane, of four tokens, whose scales for a group are four neighbouring bytes.
constexpr int kKeepCols = 512, kKeepRows = 4;

template <int GROUP, bool VEC>
__global__ __launch_bounds__(256) void k_quantize_scaled8(const KeepArgs a) {
  constexpr int kLanes = GROUP / 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = (int64_t)(blockIdx.x % a.tiles) * kKeepCols + lane * 8;
  const int64_t t0 = ((int64_t)(blockIdx.x / a.tiles) * 4 + wave) * kKeepRows;
  if (t0 >= a.T) return;  // a wave as one: lanes beyond the last column go on, their group's other lanes need them
  const int64_t left = a.K - col;
  const int n = left >= 8 ? 8 : left > 0 ? (int)left : 0;  // columns of this lane
  float v[kKeepRows][8];
#pragma unroll
  for (int r = 0; r < kKeepRows; ++r) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[r][j] = 0.0f;
    if (t0 + r < a.T && n > 0) {
      Piece q{};
      const unsigned char* row = row_of(a.x, (t0 + r) * a.ldx + col, a.x_bf16);
      if constexpr (VEC) {
        piece_load<1, true>(q, row, 0, 0, 8, a.x_bf16);
        piece_values<true>(q, a.x_bf16, v[r]);
      } else {
        piece_load<1, false>(q, row, 0, 0, n, a.x_bf16);
        piece_values<false>(q, a.x_bf16, v[r]);
      }
    }
  }
  uint32_t scales = 0;
#pragma unroll
  for (int r = 0; r < kKeepRows; ++r) {
    u32x2v codes;
    scales |= (uint32_t)quantise8<kLanes>(v[r], a.q.fmt, codes) << (8 * r);
    if (t0 + r < a.T && n > 0) {
      uint8_t* out = a.q.codes + (t0 + r) * a.q.ld + col;
      if constexpr (VEC) {
        *reinterpret_cast<u32x2v*>(out) = codes;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < n) out[j] = (uint8_t)(codes[j >> 2] >> (8 * (j & 3)));
      }
    }
  }
  if (lane % kLanes == 0 && n > 0) {
    uint8_t* s = a.q.scales + (col / GROUP) * a.q.lds + t0;
    if (t0 + kKeepRows <= a.T) {
      *reinterpret_cast<uint32_t*>(s) = scales;
    } else {
#pragma unroll
      for (int r = 0; r < kKeepRows; ++r)
        if (t0 + r < a.T) s[r] = (uint8_t)(scales >> (8 * r));
    }
  }
}

template <bool VEC>
__global__ __launch_bounds__(256) void k_dequantize_scaled8(const KeepArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = (int64_t)(blockIdx.x % a.tiles) * kKeepCols + lane * 8;
  const int64_t t0 = ((int64_t)(blockIdx.x / a.tiles) * 4 + wave) * kKeepRows;
  const int64_t left = a.K - col;
  if (left <= 0) return;
  const int n = left >= 8 ? 8 : (int)left;
#pragma unroll
  for (int r = 0; r < kKeepRows; ++r) {
    if (t0 + r >= a.T) return;
    const uint8_t* c = a.q.codes + (t0 + r) * a.q.ld + col;
    const float scale = scale_value(a.q.scales[(col >> a.q.shift) * a.q.lds + t0 + r]);  // (a lane's eight columns are of one group)
    unsigned char* row = row_of(const_cast<void*>(a.x), (t0 + r) * a.ldx + col, a.x_bf16);
    float v[8];
    if constexpr (VEC) {
      decode8(*reinterpret_cast<const u32x2v*>(c), a.q.fmt, scale, v);
      piece_store<1, true>(row, 0, 0, 8, a.x_bf16, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < n ? decode1(c[j], a.q.fmt, scale) : 0.0f;
      piece_store<1, false>(row, 0, 0, n, a.x_bf16, v);
    }
  }
}

// ---- the stored blocks of a weight, one scale each -----------------------------------------------------------------------------

template <int B>
__global__ __launch_bounds__(256) void k_quantize_blocks8(const uint16_t* vals, int fmt, uint8_t* codes, uint8_t* scales) {
  constexpr int kPieces = B * B / 8 / 256;
  __shared__ uint32_t most[4];
  const int64_t q = blockIdx.x;
  const unsigned char* in = reinterpret_cast<const unsigned char*>(vals + q * (B * B));
  float v[kPieces][8];
  Piece p[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) piece_load<256, true>(p[i], in, i, threadIdx.x, B * B, 1);
  // (finite values: a bf16 value's magnitude is at most kMostBits unless it is not finite or its largest)
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    piece_values<true>(p[i], 1, v[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t a = magnitude(v[i][j]);
      if (a < 0x7F800000u) {
        if (a > kMostBits) {
          a = kMostBits;
          v[i][j] = __builtin_copysignf(__uint_as_float(kMostBits), v[i][j]);
        }
        m = a > m ? a : m;
      }
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = __shfl_xor(m, d);
    m = o > m ? o : m;
  }
  if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) m = most[w] > m ? most[w] : m;
  const int code = scale_code(m, fmt);
  const float inv = scale_inverse(code);
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] *= inv;
    *reinterpret_cast<u32x2v*>(codes + q * (B * B) + (i * 256 + threadIdx.x) * 8) = encode8(v[i], fmt);
  }
  if (threadIdx.x == 0) scales[q] = (uint8_t)code;
}

}  // namespace blast_dev
