// Checks of blast_scaled8_view and blast_weight8_view that several calls share.
#pragma once
#include "blast_common.h"
#include "kern_scaled8.h"

namespace {

bool format8_ok(int32_t f) { return f == BLAST_E4M3 || f == BLAST_E5M2; }

// A scaled 8-bit tensor of T tokens and K features; `align`: of its codes and their pitch.
int check_eight(const blast_scaled8_view* v, int64_t T, int64_t K, int64_t align) {
  if (!v || !format8_ok(v->format) || (v->group != 64 && v->group != 128)) return BLAST_ERR_INVALID_ARG;
  if (T == 0 || K == 0) return BLAST_OK;
  if (!v->codes || v->ld < K || v->ld % align || !blast::aligned(v->codes, (size_t)align)) return BLAST_ERR_INVALID_ARG;
  if (!v->scales || v->lds < T || v->lds % 16 || !blast::aligned(v->scales, 16)) return BLAST_ERR_INVALID_ARG;
  return BLAST_OK;
}

blast_dev::Eight eight_of(const blast_scaled8_view* v) {
  return blast_dev::Eight{v->codes, v->scales, v->ld, v->lds, v->format, v->group == 64 ? 6 : 7};
}

}  // namespace
