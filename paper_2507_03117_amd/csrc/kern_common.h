// Device-side helpers shared by the product kernels.
#pragma once
#include <type_traits>

#include "blast_common.h"

namespace blast_dev {


typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct MatDev {
  const int* row_ptr;
  const int* col_idx;
  const uint16_t* vals;
  const uint8_t* vals8 = nullptr;  // E5M2 codes of the same blocks (kernels instantiated for one-byte weights)
};

struct TileArgs {
  MatDev m0, m1;         // m1 only for the dual (gate/up) kernel
  const int* row_order;  // may be null
  const uint16_t* X;
  int64_t sxt, sxk;      // element strides of X along tokens / features
  void* Y;
  int64_t syt, syi;      // element strides of Y along tokens / rows
  int y_bf16;
  int T;
  int nbr;               // block rows of the output
  int64_t kdim;          // features contracted over (columns of the matrix); host-side scheduling only
  int ntt;               // token tiles
  int act;               // gated product: the activation of the gate; single matrix: < 0 none, else applied to the output
  int x_vec;             // 1: 16-byte loads of X are legal (sxk == 1, aligned)
  int y_fast;            // 1: syi == 1 and every byte offset inside a 256-token slab of Y fits 31 bits
  int y_keep;            // E5M2 product with 128-wide blocks: 1: the output is written through the L2, else past the caches
  int y_pairs;           // 1: two neighbouring rows of a token may be stored as one value (Y and syt aligned to two values)
  int x_grp16;           // 16-wide blocks only: X is stored in column groups of 16 features, [kdim/16][T][16]
  int y_grp16;           // ... and so is Y, [rows/16][T][16]
};

// What a product with an epilogue of its own (blast_bsr_linear) does with a sum, all of it optional: Z = sum + bias, kept in
// bf16; Y = act(Z) + R.  Rows of R and Z are contiguous (token-major) where a kernel other than the generic one runs.
struct Epilogue {
  static constexpr bool kOn = true;
  const float* bias;   // per row
  const void* R;       // residual, element strides along tokens / rows
  int64_t srt, sri;
  uint16_t* Z;         // bf16
  int64_t szt, szi;
  int r_bf16;
  int act;             // BLAST_ACT_*
  int pairs, quads;    // two, four neighbouring rows of a token of R and of Z may be read / stored as one value
  // the same for the tokens from t0 on
  Epilogue from(int64_t t0) const {
    Epilogue e = *this;
    if (R) e.R = static_cast<const char*>(R) + t0 * srt * (r_bf16 ? 2 : 4);
    if (Z) e.Z = Z + t0 * szt;
    return e;
  }
};
struct NoEpilogue {
  static constexpr bool kOn = false;
  static constexpr int pairs = 1;
  NoEpilogue from(int64_t) const { return *this; }
};

// Index arrays are read-only for the lifetime of a launch: reading them through the
// constant address space lets uniform loads go through the scalar unit, so they never
// sit in the vector-memory counter that the DMA pipeline is tracked with.
__device__ __forceinline__ int ld_idx(const int* p, int i) {
  return reinterpret_cast<const __attribute__((address_space(4))) int*>(reinterpret_cast<uintptr_t>(p))[i];
}

// fp32 -> bf16, round to nearest even (the hardware conversion of gfx950).
__device__ __forceinline__ uint16_t f32_to_bf16_rne(float f) {
  const __bf16 h = static_cast<__bf16>(f);
  return __builtin_bit_cast(uint16_t, h);
}

// Stores a value of 2, 4 or 8 bytes (naturally aligned) through the L2 of this XCD to the memory side.  An output that no
// later instruction of the launch reads gains nothing from staying in the L2, and what is dirty there when the launch
// ends is written back before the next one may start: the output of a short launch then leaves while it still computes.
template <class T>
__device__ __forceinline__ void store_through(T* p, T v) {
  using U = std::conditional_t<sizeof(T) == 2, uint16_t, std::conditional_t<sizeof(T) == 4, uint32_t, unsigned long long>>;
  static_assert(sizeof(T) == sizeof(U), "two, four or eight bytes");
  __hip_atomic_store(reinterpret_cast<U*>(p), __builtin_bit_cast(U, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// g * Phi(g), Phi the normal distribution function, from its tail: Phi(-t) = 2^(t R(t)) / 2 for t = |g|, R a polynomial
// fitted to (log2 Phi(-t) + 1) / t on [0, 6] so that t times the tail's error is below 2e-9 (least squares, reweighted to
// equal ripple); its leading coefficient is negative, so the tail goes on falling beyond 6 and is 0 at infinity.  More
// accurate than 0.5 g (1 + erf(g / sqrt 2)), which rounds a sum in between (root mean square error against 64 bits over
// normal g, that with erff / this: standard deviation 0.25 5.3e-9 / 4.2e-9, 1: 2.51e-8 / 1.75e-8, 5: 6.4e-8 / 4.8e-8), in 18
// instructions without a branch, where erff has 60 in two arms, the second beyond 1.4, 64 values a lane
// (two-matrix MLP of 1600 and 6400 features at 80 %, 333 tokens: 21.1 -> 20.2 us; over 32 calls of 1024 to 4096 features and 300
// to 4096 tokens on the streaming kernel 1 % less time on average.  Rows of one or two blocks under thousands of tokens, whose
// values hardly ever need the second arm and which multiply little, take up to 4 % more: 1024 and 4096 features at 90 %, 64-wide,
// 4096 tokens 28.9 / 30.0 us).
// normal_tail: Phi(-t) for t >= 0.
__device__ __forceinline__ float normal_tail(float t) {
  float r = -5.96657159e-8f;
  r = __builtin_fmaf(r, t, 1.44687544e-6f);
  r = __builtin_fmaf(r, t, -1.56093192e-5f);
  r = __builtin_fmaf(r, t, 9.60514999e-5f);
  r = __builtin_fmaf(r, t, -3.27383575e-4f);
  r = __builtin_fmaf(r, t, 6.75653209e-5f);
  r = __builtin_fmaf(r, t, 6.89349836e-3f);
  r = __builtin_fmaf(r, t, -5.24200164e-2f);
  r = __builtin_fmaf(r, t, -4.59224194e-1f);
  r = __builtin_fmaf(r, t, -1.15110409f);
  return 0.5f * __builtin_amdgcn_exp2f(t * r);
}

__device__ __forceinline__ float gelu(float g) {
  const float t = __builtin_fabsf(g), tail = normal_tail(t);
  // max(g, 0) - |g| tail, rounded once; infinity has no tail (a finite factor), minus infinity has no value (0 g)
  return __builtin_fmaf(-__builtin_fminf(t, 3.402823466e38f), tail, g > 0.0f ? g : 0.0f * g);
}

// Activation of the output of a single product in the kernels that end with many values a lane (streaming, shared tiles).
__device__ __forceinline__ float post_act(int act, float g) {
  if (act == BLAST_ACT_SILU) return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g));
  if (act == BLAST_ACT_GELU) return gelu(g);
  return g > 0.0f ? g : 0.0f;
}

// Activation of a gated product, and of a single one in the other kernels.  It has its GELU from erff: with the shorter one beside
// the SiLU of their usual calls the kernels are laid out otherwise, and these calls are slower (16384 x 53248 at 95 % Zipf,
// 128-wide, 2048 tokens: 720 / 724 us; 4096 x 14336, 128-wide, eight layers, at 90 % 27 tokens 179 / 183 us, at 95 % 13 tokens 96
// / 100; two-matrix MLP of 2048 and 8192 features at 70 %, 32-wide, SiLU, 1 token 13.7 / 14.4, 48 tokens 18.0 / 18.8; of 1024 and
// 4096 at 90 %, 16-wide, GELU, 4096 tokens 37.6 / 38.8).
__device__ __forceinline__ float apply_act(int act, float g) {
  if (act == BLAST_ACT_SILU) return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g));
  if (act == BLAST_ACT_GELU) return 0.5f * g * (1.0f + erff(g * 0.70710678118654752440f));
  return g > 0.0f ? g : 0.0f;
}

// Activation in an Epilogue: post_act, but a NaN stays one through ReLU (the products above make it 0, as their oracle does).
__device__ __forceinline__ float epilogue_act(int act, float v) {
  if (act == BLAST_ACT_RELU) return v <= 0.0f ? 0.0f : v;
  return post_act(act, v);
}

__device__ __forceinline__ float bf16_value(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// N neighbouring rows' values (N = 1, 2, 4) of one token's residual and of the bias, asked for before they are needed: rows are
// contiguous; `wide`: the address is aligned to the N values.
template <int N>
struct EpilogueRows {
  uint32_t r[N];
  float bias[N];
};
template <int N>
__device__ __forceinline__ void epilogue_load(const Epilogue& e, EpilogueRows<N>& q, int64_t tok, int64_t row, bool wide) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    q.r[i] = 0;
    q.bias[i] = 0.0f;
  }
  if (e.bias) {
#pragma unroll
    for (int i = 0; i < N; ++i) q.bias[i] = e.bias[row + i];
  }
  if (e.R) {
    typedef uint32_t Words __attribute__((ext_vector_type(N < 2 ? 2 : N)));
    const int64_t at = tok * e.srt + row;
    if (e.r_bf16) {
      const uint16_t* p = static_cast<const uint16_t*>(e.R) + at;
      if (N > 1 && wide) {  // taken apart when they are used, or the load would be waited for here
        typedef uint32_t Pairs __attribute__((ext_vector_type(N < 4 ? 1 : N / 2)));
        const Pairs w = *reinterpret_cast<const Pairs*>(p);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) q.r[i] = w[i];
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) q.r[i] = p[i];
      }
    } else {
      const uint32_t* p = static_cast<const uint32_t*>(e.R) + at;
      if (N > 1 && wide) {
        const Words w = *reinterpret_cast<const Words*>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) q.r[i] = w[i];
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) q.r[i] = p[i];
      }
    }
  }
}
// The sums of those rows through the epilogue.
template <int N>
__device__ __forceinline__ void epilogue_apply(const Epilogue& e, const EpilogueRows<N>& q, float (&v)[N], int64_t tok, int64_t row, bool wide) {
  if (e.bias) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += q.bias[i];
  }
  if (e.Z) {
    uint16_t* p = e.Z + tok * e.szt + row;
    typedef uint16_t Halves __attribute__((ext_vector_type(N < 2 ? 2 : N)));
    if (N > 1 && wide) {
      Halves h;
#pragma unroll
      for (int i = 0; i < N; ++i) h[i] = f32_to_bf16_rne(v[i]);
      *reinterpret_cast<Halves*>(p) = h;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) p[i] = f32_to_bf16_rne(v[i]);
    }
  }
  if (e.act >= 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = epilogue_act(e.act, v[i]);
  }
  if (e.R) {
    if (N > 1 && e.r_bf16 && wide) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __uint_as_float(i % 2 ? q.r[i / 2] & 0xFFFF0000u : q.r[i / 2] << 16);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __uint_as_float(e.r_bf16 ? q.r[i] << 16 : q.r[i]);
    }
  }
}

// One value through the epilogue, in the generic kernel.  `row` counts in the whole matrix.
__device__ __forceinline__ float epilogue_value(const Epilogue& e, float v, int64_t tok, int64_t row) {
  if (e.bias) v += e.bias[row];
  if (e.Z) e.Z[tok * e.szt + row * e.szi] = f32_to_bf16_rne(v);
  if (e.act >= 0) v = epilogue_act(e.act, v);
  if (e.R) {
    const int64_t at = tok * e.srt + row * e.sri;
    v += e.r_bf16 ? bf16_value(static_cast<const uint16_t*>(e.R)[at]) : static_cast<const float*>(e.R)[at];
  }
  return v;
}

}  // namespace blast_dev
