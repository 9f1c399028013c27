// Launches of the norms' gradient.  Each kind of norm is compiled in a translation unit of its own (blast_norm_rms.hip,
// blast_norm_layer.hip): the kernels are many.
#pragma once
#include "blast_common.h"

#include "kern_norm.h"

namespace blast {

// Workgroups of a backward pass, each with column sums of its own: one to a row up to kBackwardRows rows, beyond that one of
// sixteen waves per CU of the full card.  From the sizes alone, so that the workspace does not depend on the device.
// One number for both forms of few rows, where the two would have different ones.  GPU time from a graph, microseconds, a row to a
// workgroup / workgroups that go over the rows, bf16:
//     columns with owners, RMS:        1600 features, 333 rows 5.5 / 9.3, 512: 7.1 / 8.7, 1024: 11.9 / 10.6; 4096, 512: 8.5 / 12.2, 1024: 13.1 /
//       15.2; 16384, 333: 20.8 / 21.4, 512: 27.5 / 25.4; 512 features, 257: 7.9 / 7.6, 512: 12.2 / 7.9 (few owners)
//     rows' sums joined, RMS on both sides, gate of one row: 512 features, 333 rows 8.9 / 9.3; 1600, 257: 10.0 / 10.5, 333: 12.8 / 11.1; 4096,
//       257: 16.4 / 13.6, 512: 20.2 / 17.3; 16384, 257: 42 / 42, 512: 66 / 52
constexpr int kBackwardRows = 512, kBackwardGroups = 256;

// Few rows: the columns have workgroups of their own in the launch of the rows, instead of a second launch that joins the rows'
// sums, where no other sums are wanted than those of the norm of the stream.
inline bool columns_owned(int64_t T, bool branch, int post, bool gate_of_one_row) {
  return T <= kBackwardRows && (!branch || (!post && !gate_of_one_row));
}

// The launches of a call whose arguments have been checked; `vec`: every operand takes 16-byte access.
int norm_backward_rms(const blast_dev::NormArgs& a, bool vec, hipStream_t stream);
int norm_backward_layer(const blast_dev::NormArgs& a, bool vec, hipStream_t stream);

}  // namespace blast

namespace {

using namespace blast_dev;
using blast::kBackwardGroups;
using blast::kBackwardRows;

template <int NW, int NCH, int TEAMS, bool VEC, bool LOOP, bool ROOM, bool LOW, bool COLS, bool LAYER, int MODE>
int launch_backward_m(NormArgs a, hipStream_t stream) {
  constexpr int kThreads = 64 * NW * TEAMS, kSums = 1 + (MODE >= 1) + LAYER + (LAYER && MODE == 2);
  constexpr size_t kSumBytes = (size_t)kThreads * NCH * 8 * 4;
  // sums in LDS: as many as fit, the workgroup having a CU to itself; none where it has one row
  constexpr int kFit = (int)((size_t)(150 << 10) / kSumBytes), NL = !LOOP ? 0 : kSums < kFit ? kSums : kFit;
  constexpr size_t kLds = (size_t)NL * kSumBytes;
  constexpr bool AHEAD = LOOP && ROOM && !(NCH > 1 && LAYER && MODE >= 1);  // (two sums of a layer norm are then in registers)
  const int64_t rows = (a.T + TEAMS - 1) / TEAMS;
  int64_t grid = LOOP && rows > kBackwardGroups ? kBackwardGroups : rows;
  if constexpr (COLS) {
    if (a.sum_out[0] || a.sum_out[1]) a.column_groups = (a.width + 16 * kNormOwned - 1) / (16 * kNormOwned) * 16;
    grid += a.column_groups;
  }
  constexpr auto kernel = &k_norm_backward<NW, NCH, TEAMS, VEC, LAYER, MODE, NL, LOOP, AHEAD, LOW, COLS>;
  if constexpr (kLds > 48 * 1024) {
    static blast::DeviceFlags lds_set;
    int dev = 0;
    BLAST_HIP_TRY(hipGetDevice(&dev));
    if (!lds_set.test(dev)) {
      BLAST_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds));
      lds_set.set(dev);
    }
  }
  kernel<<<dim3((unsigned)grid), dim3(kThreads), kLds, stream>>>(a);
  BLAST_LAUNCH_CHECK("k_norm_backward");
  if (COLS || grid == 1) return BLAST_OK;
  JoinArgs j{};
  j.part = a.part;
  j.groups = (int)grid;
  j.width = a.width;
  int n = 0;
  for (int s = 0; s < kNormSums; ++s)
    if (a.sum_out[s]) j.out[n++] = a.sum_out[s];
  if (n == 0) return BLAST_OK;
  k_join_sums<<<dim3((unsigned)((a.width + 63) / 64), (unsigned)n), dim3(1024), 0, stream>>>(j);
  BLAST_LAUNCH_CHECK("k_join_sums");
  return BLAST_OK;
}

template <bool LAYER, int NW, int NCH, int TEAMS, bool VEC, bool LOOP, bool ROOM, bool LOW = false>
int launch_backward(const NormArgs& a, hipStream_t stream) {
  const int mode = !a.y ? 0 : a.post ? 2 : 1;
  if constexpr (!LOOP) {
    if (blast::columns_owned(a.T, a.y != nullptr, a.post, a.gate && a.ldg == 0)) {
      if (mode == 0) return launch_backward_m<NW, NCH, TEAMS, VEC, false, false, LOW, true, LAYER, 0>(a, stream);
      return launch_backward_m<NW, NCH, TEAMS, VEC, false, false, LOW, true, LAYER, 1>(a, stream);
    }
  } else {
    if (mode == 0) return launch_backward_m<NW, NCH, TEAMS, VEC, true, ROOM, LOW, false, LAYER, 0>(a, stream);
  }
  if (mode == 1) return launch_backward_m<NW, NCH, TEAMS, VEC, LOOP, ROOM, LOW, false, LAYER, 1>(a, stream);
  return launch_backward_m<NW, NCH, TEAMS, VEC, LOOP, ROOM, LOW, false, LAYER, 2>(a, stream);
}

template <bool LAYER>
int dispatch_backward(const NormArgs& a, bool vec, hipStream_t stream) {
  const bool few = a.T <= kBackwardRows;  // a row to a workgroup
  if (!vec) {
    if (a.width <= 2048)
      return few ? launch_backward<LAYER, 4, 1, 1, false, false, false>(a, stream)
                 : launch_backward<LAYER, 4, 1, 1, false, true, false>(a, stream);
    if (a.width <= 8192)
      return few ? launch_backward<LAYER, 16, 1, 1, false, false, false>(a, stream)
                 : launch_backward<LAYER, 16, 1, 1, false, true, false>(a, stream);
    return few ? launch_backward<LAYER, 16, 4, 1, false, false, false>(a, stream)
               : launch_backward<LAYER, 16, 4, 1, false, true, false>(a, stream);
  }
  const bool low = a.h_bf16 && a.dx_bf16 && (!a.w || a.p_bf16) &&
                   (!a.y || (a.y_bf16 && (!a.dy || a.dy_bf16) && (!a.gate || a.g_bf16) && ((!a.pw && !a.pb) || a.p_bf16)));
  if (few) {
    if (a.width <= 512) return launch_backward<LAYER, 1, 1, 1, true, false, false>(a, stream);
    if (a.width <= 1024) return launch_backward<LAYER, 2, 1, 1, true, false, false>(a, stream);
    if (a.width <= 2048) return launch_backward<LAYER, 4, 1, 1, true, false, false>(a, stream);
    if (a.width <= 4096) return launch_backward<LAYER, 8, 1, 1, true, false, false>(a, stream);
    if (a.width <= 8192) return launch_backward<LAYER, 16, 1, 1, true, false, false>(a, stream);
    if (a.width <= 16384)
      return low ? launch_backward<LAYER, 16, 2, 1, true, false, false, true>(a, stream)
                 : launch_backward<LAYER, 16, 2, 1, true, false, false>(a, stream);
    return launch_backward<LAYER, 16, 4, 1, true, false, false>(a, stream);
  }
  if (a.width <= 512) return launch_backward<LAYER, 1, 1, 16, true, true, true>(a, stream);
  if (a.width <= 1024) return launch_backward<LAYER, 2, 1, 8, true, true, true>(a, stream);
  if (a.width <= 2048) return launch_backward<LAYER, 4, 1, 4, true, true, true>(a, stream);
  if (a.width <= 4096) return launch_backward<LAYER, 8, 1, 2, true, true, true>(a, stream);
  if (a.width <= 8192) return launch_backward<LAYER, 16, 1, 1, true, true, true>(a, stream);
  if (a.width <= 16384)
    return low ? launch_backward<LAYER, 16, 2, 1, true, true, true, true>(a, stream)
               : launch_backward<LAYER, 16, 2, 1, true, true, false>(a, stream);
  return launch_backward<LAYER, 16, 4, 1, true, true, false>(a, stream);
}

}  // namespace
