// Row-wise kernels' common parts: a row's values as 8-value pieces held in registers, sums over the lanes that share a row,
// and the joining of per-workgroup column sums.
#pragma once
#include "kern_common.h"

namespace blast_dev {

// Eight values of a row as they lie in memory: bf16 pairs in the first four words or fp32 values; with element-wise access
// one value a word.  They are converted only when they are used: loads of several tensors are then all on their way before
// the first is waited for, whatever their types (the types are the same for all lanes: the branches are scalar).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
struct Piece {
  u32x4 lo, hi;
};

// Element j of piece c of lane `lane` of the NT lanes that share a row: VEC keeps a lane's eight together, so that a lane
// reads 16 or 32 bytes; element-wise access (any width, pitch and alignment) puts neighbouring lanes on neighbouring elements.
template <int NT, bool VEC>
__device__ __forceinline__ int piece_at(int c, int j, int lane) {
  return VEC ? (c * NT + lane) * 8 + j : (c * 8 + j) * NT + lane;
}

// A row of a tensor: where it is the same for all lanes of a wave, an access is a scalar base and a lane's 32-bit offset.
__device__ __forceinline__ const unsigned char* row_of(const void* base, int64_t at, int bf16) {
  return static_cast<const unsigned char*>(base) + (bf16 ? at * 2 : at * 4);
}
__device__ __forceinline__ unsigned char* row_of(void* base, int64_t at, int bf16) {
  return static_cast<unsigned char*>(base) + (bf16 ? at * 2 : at * 4);
}

// Four values that are the same for all lanes and that the launch does not write, through the scalar unit.
__device__ __forceinline__ float4 scalar_float4(const float* p) {
  const auto* q = reinterpret_cast<const __attribute__((address_space(4))) float*>(reinterpret_cast<uintptr_t>(p));
  return float4{q[0], q[1], q[2], q[3]};
}

template <int NT, bool VEC>
__device__ __forceinline__ void piece_load(Piece& q, const unsigned char* row, int c, int lane, int width, int bf16) {
  if constexpr (VEC) {
    const uint32_t e = (uint32_t)(c * NT + lane) * 8;
    if (e < (uint32_t)width) {
      if (bf16) {
        q.lo = *reinterpret_cast<const u32x4*>(row + e * 2);
      } else {
        const u32x4* p = reinterpret_cast<const u32x4*>(row + e * 4);
        q.lo = p[0];
        q.hi = p[1];
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t e = (uint32_t)((c * 8 + j) * NT + lane);
      uint32_t v = 0;
      if (e < (uint32_t)width) v = bf16 ? *reinterpret_cast<const uint16_t*>(row + e * 2) : *reinterpret_cast<const uint32_t*>(row + e * 4);
      if (j < 4)
        q.lo[j & 3] = v;
      else
        q.hi[j & 3] = v;
    }
  }
}

template <bool VEC>
__device__ __forceinline__ void piece_values(const Piece& q, int bf16, float (&out)[8]) {
  auto word = [&](int i) { return i < 4 ? q.lo[i & 3] : q.hi[i & 3]; };
  if (bf16) {
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = __uint_as_float(!VEC ? word(j) << 16 : j % 2 ? word(j / 2) & 0xFFFF0000u : word(j / 2) << 16);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = __uint_as_float(word(j));
  }
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  return (uint32_t)f32_to_bf16_rne(a) | ((uint32_t)f32_to_bf16_rne(b) << 16);
}

// PAST: the result leaves past the L2 (see kPastBytes).
template <int NT, bool VEC, bool PAST = false>
__device__ __forceinline__ void piece_store(unsigned char* row, int c, int lane, int width, int bf16, const float (&v)[8]) {
  if constexpr (VEC) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    auto put = [](auto* p, auto x) {
      if constexpr (PAST)
        __builtin_nontemporal_store(x, p);
      else
        *p = x;
    };
    const uint32_t e = (uint32_t)(c * NT + lane) * 8;
    if (e < (uint32_t)width) {
      if (bf16) {
        put(reinterpret_cast<u32x4*>(row + e * 2),
            u32x4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])});
      } else {
        f32x4* p = reinterpret_cast<f32x4*>(row + e * 4);
        put(p, f32x4{v[0], v[1], v[2], v[3]});
        put(p + 1, f32x4{v[4], v[5], v[6], v[7]});
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t e = (uint32_t)((c * 8 + j) * NT + lane);
      if (e < (uint32_t)width) {
        if (bf16)
          *reinterpret_cast<uint16_t*>(row + e * 2) = f32_to_bf16_rne(v[j]);
        else
          *reinterpret_cast<float*>(row + e * 4) = v[j];
      }
    }
  }
}

// Sum over the wave, in every lane: shifts inside rows of 16 lanes, then the rows' totals passed on, then lane 63's.
__device__ __forceinline__ float wave_sum(float x) {
  auto add = [&](auto ctrl, auto rows) {
    x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl.value, rows.value, 0xF, true));
  };
  add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xF>{});
  add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xF>{});
  add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xF>{});
  add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xF>{});
  add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});
  add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// Sums of N values over the NW waves that share a row.  The waves' sums meet in LDS and are added in wave order by every
// wave.  Two buffers take turns: a wave that writes one again has passed the barrier of the other, and every wave had read
// this one by then.
template <int NW>
struct RowSum {
  float (*buf)[NW][2];
  int wave;  // of the row's NW
  int turn = 0;
  template <int N>
  __device__ __forceinline__ void operator()(float (&s)[N]) {
    static_assert(N <= 2, "");
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
    if constexpr (NW > 1) {
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) buf[turn][wave][i] = s[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float t = buf[turn][0][i];
#pragma unroll
        for (int w = 1; w < NW; ++w) t += buf[turn][w][i];
        s[i] = t;
      }
      turn ^= 1;
    }
  }
};

// out[s][e] = sum over g of part[(s * groups + g) * width + e]: the column sums of the workgroups of an earlier launch.  A
// workgroup takes 64 columns of one sum, its 16 waves every 16th group, whose sums meet in LDS in a fixed order.
struct JoinArgs {
  const float* part;
  float* out[5];
  int groups, width;
};
static __global__ __launch_bounds__(1024) void k_join_sums(const JoinArgs a) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = (int)blockIdx.x * 64 + lane, s = blockIdx.y;
  const float* p = a.part + (int64_t)s * a.groups * a.width + e;
  float v = 0.0f;
  if (e < a.width) {
#pragma unroll 8
    for (int g = wave; g < a.groups; g += 16) v += p[(int64_t)g * a.width];
  }
  red[wave][lane] = v;
  __syncthreads();
  if (wave == 0 && e < a.width) {
    float t = red[0][lane];
#pragma unroll
    for (int w = 1; w < 16; ++w) t += red[w][lane];
    a.out[s][e] = t;
  }
}

// Zeros for the column sums over no rows.
static __global__ __launch_bounds__(256) void k_zero_sums(const JoinArgs a) {
  const int e = (int)blockIdx.x * 256 + threadIdx.x;
  if (e < a.width) a.out[blockIdx.y][e] = 0.0f;
}

}  // namespace blast_dev
