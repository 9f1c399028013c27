// Launches of the block-sparse products and the host rules that pick a kernel, shared by the translation units that
// instantiate them: blast_spmm.hip (products, MLP) and blast_linear.hip (the product with an epilogue of its own).
#pragma once
#include "blast_common.h"

#include <atomic>
#include <cmath>

#include "kern_common.h"
#include "kern_tile.h"
#include "kern_stream.h"
#include "kern_decode.h"
#include "kern_flat.h"
#include "kern_b16.h"
#include "kern_split.h"

using namespace blast_dev;

namespace {

// Raises a kernel's dynamic-LDS limit once per device (the attribute is per device; setting it again
// is harmless, so a race between host threads only repeats the call).
int ensure_lds_limit(const void* kernel, size_t bytes, blast::DeviceFlags& done) {
  int dev = 0;
  BLAST_HIP_TRY(hipGetDevice(&dev));
  if (done.test(dev)) return BLAST_OK;
  BLAST_HIP_TRY(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
  done.set(dev);
  return BLAST_OK;
}

template <int B, bool DUAL, class EPI = NoEpilogue>
int launch_tile(TileArgs a, hipStream_t stream, const EPI& epi = EPI{}) {
  using C = TileCfg<B>;
  a.ntt = (a.T + C::TT - 1) / C::TT;
  const int64_t grid = (int64_t)a.ntt * a.nbr;
  if (grid <= 0) return BLAST_OK;
  if (grid > INT32_MAX) return BLAST_ERR_INVALID_ARG;
  if constexpr (!DUAL && !EPI::kOn) {
    if (a.act >= 0) {  // single matrix with an activation on the output
      static blast::DeviceFlags lds_set_post;
      if (int rc = ensure_lds_limit(reinterpret_cast<const void*>(&k_spmm_tile<B, false, true>), C::LDS_BYTES, lds_set_post))
        return rc;
      k_spmm_tile<B, false, true><<<dim3((unsigned)grid), dim3(256), C::LDS_BYTES, stream>>>(a, epi);
      BLAST_LAUNCH_CHECK("k_spmm_tile");
      return BLAST_OK;
    }
  }
  static blast::DeviceFlags lds_set;
  if (int rc = ensure_lds_limit(reinterpret_cast<const void*>(&k_spmm_tile<B, DUAL, false, EPI>), C::LDS_BYTES, lds_set)) return rc;
  k_spmm_tile<B, DUAL, false, EPI><<<dim3((unsigned)grid), dim3(256), C::LDS_BYTES, stream>>>(a, epi);
  BLAST_LAUNCH_CHECK("k_spmm_tile");
  return BLAST_OK;
}

// 16 x 16 blocks, token-major 16-byte-aligned activations: pairs of blocks on the 32-deep matrix instruction,
// operands straight from global memory.  A wave takes 16, 32 or 64 tokens of one block row.
int cu_count();

template <bool DUAL, bool POST, int NS, bool SPLIT, int NW = 4, int DEPTH = 0, class EPI = NoEpilogue>
int launch_b16_ns(TileArgs a, int y_vec, hipStream_t stream, const EPI& epi) {
  a.ntt = (a.T + 16 * NS - 1) / (16 * NS);
  const int64_t items = (int64_t)a.ntt * a.nbr;
  const int64_t grid = SPLIT ? items : (items + 3) / 4;
  if (grid <= 0) return BLAST_OK;
  if (grid > INT32_MAX) return BLAST_ERR_INVALID_ARG;
  k_spmm_b16<DUAL, POST, NS, SPLIT, NW, DEPTH, EPI><<<dim3((unsigned)grid), dim3(NW * 64), 0, stream>>>(a, y_vec, epi);
  BLAST_LAUNCH_CHECK("k_spmm_b16");
  return BLAST_OK;
}

// A wave takes 16, 32 or 64 tokens of a block row.  While that makes fewer than eight waves per CU, a workgroup
// shares one (block row, token tile) and its waves deal the row's blocks: 1B-shaped layer, 128 tokens,
// 31 -> 19 us per MLP pass, 512 tokens 39 -> 32.  Up to 16 tokens, rows of more than 16 pairs on average go to
// sixteen waves instead of four (the 1B-shaped down projection: 128 rows of 51 blocks).
template <bool DUAL, bool POST, class EPI>
int launch_b16_t(const TileArgs& a, int64_t nnz, int y_vec, hipStream_t stream, const EPI& epi) {
  if (a.T <= 16) {
    if (nnz > (int64_t)32 * a.nbr) return launch_b16_ns<DUAL, POST, 1, true, 16>(a, y_vec, stream, epi);
    return launch_b16_ns<DUAL, POST, 1, true>(a, y_vec, stream, epi);
  }
  if (a.T <= 32) return launch_b16_ns<DUAL, POST, 2, true>(a, y_vec, stream, epi);
  const bool split = (int64_t)((a.T + 63) / 64) * a.nbr < 8 * cu_count();
  // (column groups that 32-bit byte offsets reach, a wave's 64 tokens past the end included)
  if (a.x_grp16 && ((int64_t)a.kdim / 16 * a.T + 64) * 32 < ((int64_t)1 << 32)) {
    // Two pairs in flight, or one.  While 64-token tiles divide the 32 that the eight XCDs take in four-wave workgroups, the
    // workgroups of an XCD keep to the same tokens, whose activations stay in its L2, and what is left is latency: two.
    // Otherwise every XCD goes over all tokens, and more in flight only pushes activations out of the L2 before the next row
    // reads them: one, unless there are few tokens or, with shared rows, no second workgroup on a CU.  Microseconds, walk of `b16_row` / two / one: 2048 x 8192 at 70 %, 1024
    // tokens 56.9 / 44.0 / 46.5, 2048: 79.7 / 78.0 / 83.3; 1280: 66.8 / 76.2 / 72.1, 2500: 135 / 145 / 100, 4096: 157 / 167 /
    // 146; 4096 x 4096 at 90 %, 1280: 34.5 / 38.7 / 35.0; 1024 x 16384 at 70 %, 700 tokens (split) 53.6 / 63.0 / 54.2, 2500: 149
    // / 181 / 165; 512 x 8192 at 70 %, 300 (split) 21.2 / 16.5 / 18.6; MLP of 2048 and 8192 features at 90 %, 333 tokens 29.9 / 27.9 / 28.8, 500: 31.9 / 30.5 / 32.3.
    const int tiles = (a.T + 63) / 64;
    const bool two = (tiles <= 32 && 32 % tiles == 0) || (split ? (int64_t)tiles * a.nbr <= cu_count() : tiles <= 8);
    if (split)
      return two ? launch_b16_ns<DUAL, POST, 4, true, 4, 2>(a, y_vec, stream, epi) : launch_b16_ns<DUAL, POST, 4, true, 4, 1>(a, y_vec, stream, epi);
    return two ? launch_b16_ns<DUAL, POST, 4, false, 4, 2>(a, y_vec, stream, epi) : launch_b16_ns<DUAL, POST, 4, false, 4, 1>(a, y_vec, stream, epi);
  }
  if (split) return launch_b16_ns<DUAL, POST, 4, true>(a, y_vec, stream, epi);
  return launch_b16_ns<DUAL, POST, 4, false>(a, y_vec, stream, epi);
}

template <bool DUAL, class EPI>
int launch_b16(const TileArgs& a, int64_t nnz, hipStream_t stream, const EPI& epi) {
  const int y_vec = a.y_grp16 || (a.syi == 1 && a.syt % 4 == 0 && blast::aligned(a.Y, a.y_bf16 ? 8 : 16));
  if constexpr (!DUAL && !EPI::kOn) {
    if (a.act >= 0) return launch_b16_t<false, true>(a, nnz, y_vec, stream, epi);  // an activation on the output
  }
  return launch_b16_t<DUAL, false>(a, nnz, y_vec, stream, epi);
}

// From this many tokens on, a product with 16-wide blocks reads its activations from column groups of 16
// features ([K/16][T][16], see kern_b16.h) when the caller's workspace has room for the regrouped copy.
constexpr int64_t kGroup16MinTokens = 33;
size_t group16_bytes(int64_t K, int64_t T) { return blast::align_up((size_t)K * (size_t)T * 2, 256); }
bool group16_applies(int32_t b, int32_t x_layout, const void* X, int64_t ldx, int64_t T) {
  return b == 16 && T >= kGroup16MinTokens && x_layout == BLAST_TOKEN_MAJOR && ldx % 8 == 0 && blast::aligned(X, 16);
}
int enqueue_group16(const uint16_t* X, int64_t ldx, int64_t T, int64_t K, uint16_t* Xg, hipStream_t stream) {
  const int64_t nbc = K / 16;
  if (T <= 0 || nbc <= 0) return BLAST_OK;
  if ((nbc + 7) / 8 > 65535) return BLAST_ERR_INVALID_ARG;
  k_group16<<<dim3((unsigned)((T + 15) / 16), (unsigned)((nbc + 7) / 8)), dim3(256), 0, stream>>>(X, ldx, (int)T, (int)nbc, Xg);
  BLAST_LAUNCH_CHECK("k_group16");
  return BLAST_OK;
}

int cu_count() {
  static std::atomic<int> cached[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    cached[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

// Rows of an fp32 output that a later chunked product accumulates into; a launch before it can clear them
// on the side (see DecArgs) and says so in `done`.
struct ZeroJob {
  const int* hdr = nullptr;
  const int* chunk_row = nullptr;
  const int* chunk_kb = nullptr;
  const int* row_ptr = nullptr;
  float* Y = nullptr;
  int64_t syt = 0, syi = 0;
  int T = 0;
  int64_t max_chunks = 0;
  bool wide = false;  // the plan is the one of kWideChunkBlocks (its cut rows are a subset of the other plan's)
  bool done = false;
};

// Chunk plan of a packed matrix, as pointers into its aux buffer (null when it is not to be used).
struct ChunkPlan {
  const int* hdr = nullptr;
  const int* chunk_row = nullptr;
  const int* chunk_kb = nullptr;
  const int* chunk_ke = nullptr;
  int64_t max_chunks = 0;  // host-side upper bound of hdr[0]
  // the same rows in chunks of kWideChunkBlocks, for the streaming kernels
  const int* w_hdr = nullptr;
  const int* w_chunk_row = nullptr;
  const int* w_chunk_kb = nullptr;
  const int* w_chunk_ke = nullptr;
  int64_t w_max_chunks = 0;
  int max_row_blocks = 0;  // stored blocks of the fullest block row
  int64_t fullest = 0;     // the same of a single matrix, also where there is no plan (a hint; 0: not known)
  ZeroJob* zero_job = nullptr;  // a side job this launch may take along (decode launches: the first plan's only)
  bool pre_zeroed = false;      // the shared rows of the output have been cleared by an earlier launch ...
  bool zeroed_wide = false;     // ... those of the wide plan only (a subset of the other plan's)
  bool stream_narrow = false;   // the streaming kernels take the chunks of kChunkBlocks too (few token tiles)
  // long rows of a gated product cut into chunks (see StreamArgs)
  const int* slot0 = nullptr;
  const int* slot1 = nullptr;
  const int* chunk0_0 = nullptr;
  const int* chunk0_1 = nullptr;
  float* P0 = nullptr;
  float* P1 = nullptr;
  float* W0 = nullptr;
  float* W1 = nullptr;
  const int* hdr1 = nullptr;  // the second matrix' plan (the first one's is hdr, chunk_*)
  const int* chunk_row1 = nullptr;
  const int* chunk_kb1 = nullptr;
  const int* chunk_ke1 = nullptr;
  int64_t max_chunks1 = 0;
};

template <int B, bool DUAL, int TW, bool CHUNK, int NW = 4, bool LONG = false, class EPI = NoEpilogue>
int launch_stream_tw(TileArgs a, const ChunkPlan& plan, int64_t k_features, hipStream_t stream, const EPI& epi = EPI{}) {
  using C = StreamCfg<B, TW, NW>;
  a.ntt = (a.T + C::TT - 1) / C::TT;
  const int64_t n_rows = CHUNK ? plan.max_chunks : (int64_t)a.nbr + (LONG ? plan.max_chunks + plan.max_chunks1 : 0);
  const int64_t n_items = (int64_t)a.ntt * n_rows;
  if (n_items <= 0) return BLAST_OK;
  if (n_items > INT32_MAX / 2) return BLAST_ERR_INVALID_ARG;
  StreamArgs sa{};
  sa.t = a;
  sa.hdr = plan.hdr;
  sa.chunk_row = plan.chunk_row;
  sa.chunk_kb = plan.chunk_kb;
  sa.chunk_ke = plan.chunk_ke;
  const int64_t slab = ((int64_t)a.ntt + 7) / 8 * C::TT * k_features * 2;
  const int64_t grid = stream_grid<C, B>(sa, n_rows, cu_count(), slab);
  if constexpr (LONG) {
    sa.hdr1 = plan.hdr1;
    sa.chunk_row1 = plan.chunk_row1;
    sa.chunk_kb1 = plan.chunk_kb1;
    sa.chunk_ke1 = plan.chunk_ke1;
    sa.slot0 = plan.slot0;
    sa.slot1 = plan.slot1;
    sa.chunk0_0 = plan.chunk0_0;
    sa.chunk0_1 = plan.chunk0_1;
    sa.P0 = plan.P0;
    sa.P1 = plan.P1;
    sa.W0 = plan.W0;
    sa.W1 = plan.W1;
  }
  if (!CHUNK && plan.zero_job && plan.zero_job->hdr && !plan.zero_job->done) {
    // a later chunked product's rows are cleared by this launch on the side
    ZeroJob& z = *plan.zero_job;
    sa.z_hdr = z.hdr;
    sa.z_chunk_row = z.chunk_row;
    sa.z_chunk_kb = z.chunk_kb;
    sa.z_row_ptr = z.row_ptr;
    sa.z_Y = z.Y;
    sa.z_syt = z.syt;
    sa.z_syi = z.syi;
    sa.z_T = z.T;
    z.done = true;
  }
  if constexpr (CHUNK) {
    if (!plan.pre_zeroed) {
      k_zero_shared_rows<B><<<dim3((unsigned)plan.max_chunks, (unsigned)((a.T + 63) / 64)), dim3(256), 0, stream>>>(sa);
      BLAST_LAUNCH_CHECK("k_zero_shared_rows");
    }
  }
  auto launch = [&](auto post, auto pairs) -> int {
    constexpr auto kernel = &k_spmm_stream<B, DUAL, TW, CHUNK, post.value, NW, LONG, false, pairs.value, EPI>;
    static blast::DeviceFlags lds_set;
    if (int rc = ensure_lds_limit(reinterpret_cast<const void*>(kernel), C::LDS_BYTES, lds_set)) return rc;
    kernel<<<dim3((unsigned)grid), dim3(64 * NW), C::LDS_BYTES, stream>>>(sa, epi);
    BLAST_LAUNCH_CHECK("k_spmm_stream");
    return BLAST_OK;
  };
  if constexpr (!DUAL && !CHUNK && !LONG && !EPI::kOn) {
    // single matrix with an activation on the output: the intermediate of a two-matrix MLP, which takes row pairs
    if (a.act >= 0) return launch(std::true_type{}, std::true_type{});
  }
  int rc;
  if constexpr (C::PAIR && !CHUNK && !LONG)
    // Two rows to a store: only where Y (and what an epilogue reads and keeps) allows it, and with 128-wide blocks not in fp32, where whole lines leave either way (14336
    // x 4096 at 90 %, pairs / neighbouring rows, 512 tokens 19.4 / 18.9 us, 2048: 46.0 / 45.0; 53248 x 16384 at 95 %, 300: 64.2 / 62.5).
    rc = a.y_fast && a.y_pairs && epi.pairs && !(B == 128 && !a.y_bf16) ? launch(std::false_type{}, std::true_type{}) : launch(std::false_type{}, std::false_type{});
  else
    rc = launch(std::false_type{}, std::true_type{});
  if (rc) return rc;
  if constexpr (LONG) {
    k_long_finish<B><<<dim3((unsigned)((a.nbr + kLongFinishRows - 1) / kLongFinishRows),
                            (unsigned)((a.T + kLongFinishTokens - 1) / kLongFinishTokens)),
                       dim3(256), 0, stream>>>(sa);
    BLAST_LAUNCH_CHECK("k_long_finish");
  }
  return BLAST_OK;
}

template <int B, bool DUAL, bool CHUNK, class EPI = NoEpilogue>
int launch_stream_c(const TileArgs& a, const ChunkPlan& plan, int64_t k_features, hipStream_t stream, const EPI& epi = EPI{}) {
  if constexpr (B == 128) {
    // 256-token x 128-row tiles (eight waves, one workgroup per CU) once every CU gets at least two of them;
    // below that, 128-token tiles in four-wave workgroups, two per CU (8B-shaped down projection at 2048
    // tokens, 256 wide tiles: 24.9 against 28.2 us)
    const int64_t n_rows = CHUNK ? plan.max_chunks : (int64_t)a.nbr;
    const int64_t wide_items = (int64_t)((a.T + 255) / 256) * n_rows;
    if (wide_items >= 2 * (int64_t)cu_count())
      return launch_stream_tw<B, DUAL, 4, CHUNK, 8, false>(a, plan, k_features, stream, epi);
    return launch_stream_tw<B, DUAL, 2, CHUNK, 4, false>(a, plan, k_features, stream, epi);
  } else if constexpr (B == 64) {
    // 128-token tiles when 256-token tiles would leave workgroup slots empty
    const int64_t wide_items = (int64_t)((a.T + 255) / 256) * a.nbr;
    if (wide_items < (int64_t)cu_count() * 2)
      return launch_stream_tw<B, DUAL, 2, CHUNK, 4, false>(a, plan, k_features, stream, epi);
    return launch_stream_tw<B, DUAL, 4, CHUNK, 4, false>(a, plan, k_features, stream, epi);
  } else {
    return launch_stream_tw<B, DUAL, 4, CHUNK, 4, false>(a, plan, k_features, stream, epi);
  }
}

template <int B, bool DUAL, class EPI>
int launch_stream(const TileArgs& a, const ChunkPlan& plan, int64_t k_features, hipStream_t stream, const EPI& epi) {
  if constexpr (!DUAL && !EPI::kOn) {
    // rows cut into chunks accumulate with fp32 atomics: only for fp32 output without an activation
    if (plan.hdr && plan.stream_narrow && !a.y_bf16 && a.act < 0) {
      ChunkPlan narrow{};
      narrow.hdr = plan.hdr;
      narrow.chunk_row = plan.chunk_row;
      narrow.chunk_kb = plan.chunk_kb;
      narrow.chunk_ke = plan.chunk_ke;
      narrow.max_chunks = plan.max_chunks;
      narrow.max_row_blocks = plan.max_row_blocks;
      narrow.pre_zeroed = plan.pre_zeroed && !plan.zeroed_wide;
      return launch_stream_c<B, false, true>(a, narrow, k_features, stream);
    }
    if (plan.w_hdr && !a.y_bf16 && a.act < 0) {
      ChunkPlan wide{};
      wide.hdr = plan.w_hdr;
      wide.chunk_row = plan.w_chunk_row;
      wide.chunk_kb = plan.w_chunk_kb;
      wide.chunk_ke = plan.w_chunk_ke;
      wide.max_chunks = plan.w_max_chunks;
      wide.max_row_blocks = plan.max_row_blocks;
      wide.pre_zeroed = plan.pre_zeroed;  // either plan's rows cleared covers these
      return launch_stream_c<B, false, true>(a, wide, k_features, stream);
    }
  }
  ChunkPlan side{};  // no chunks; only the side job travels on
  side.zero_job = plan.zero_job;
  return launch_stream_c<B, DUAL, false>(a, side, k_features, stream, epi);
}

// Few output tiles: a workgroup per (64 rows of a block row, 64 tokens), see kern_split.h.
template <int B, int NWAVES, class EPI>
int launch_split(const TileArgs& a, hipStream_t stream, const EPI& epi) {
  using C = SplitCfg<B, NWAVES>;
  const int64_t units = (int64_t)a.nbr * C::SUB, groups = (a.T + C::SB - 1) / C::SB;
  const int64_t grid = split_workgroups(units, groups, cu_count());
  if (grid <= 0) return BLAST_OK;
  if (grid > INT32_MAX) return BLAST_ERR_INVALID_ARG;
  auto launch = [&](auto post) {
    static blast::DeviceFlags lds_set;
    if (int rc = ensure_lds_limit(reinterpret_cast<const void*>(&k_spmm_split<B, post.value, NWAVES, EPI>), C::LDS_BYTES, lds_set)) return rc;
    k_spmm_split<B, post.value, NWAVES, EPI><<<dim3((unsigned)grid), dim3(64 * C::NW), C::LDS_BYTES, stream>>>(
        a, (int)units, (int)groups, split_stride_log2(units, groups, cu_count()), epi);
    BLAST_LAUNCH_CHECK("k_spmm_split");
    return (int)BLAST_OK;
  };
  if constexpr (EPI::kOn)
    return launch(std::false_type{});
  else
    return a.act >= 0 ? launch(std::true_type{}) : launch(std::false_type{});
}

template <int B, bool DUAL, int NTT, bool CHUNK, int XSMALL, class EPI = NoEpilogue>
int launch_decode_ntt(const TileArgs& a, const ChunkPlan& plan, hipStream_t stream, const EPI& epi = EPI{}) {
  DecArgs d{};
  d.m0 = a.m0;
  d.m1 = a.m1;
  d.row_order = a.row_order;
  d.X = a.X;
  d.sxt = a.sxt;
  d.Y = a.Y;
  d.syt = a.syt;
  d.syi = a.syi;
  d.y_bf16 = a.y_bf16;
  d.T = a.T;
  d.act = a.act;
  d.hdr = plan.hdr;
  d.chunk_row = plan.chunk_row;
  d.chunk_kb = plan.chunk_kb;
  d.chunk_ke = plan.chunk_ke;
  const int64_t units = (CHUNK ? plan.max_chunks : (int64_t)a.nbr) * (B / 16);
  if (units <= 0) return BLAST_OK;
  const int64_t groups = (a.T + NTT * 16 - 1) / (NTT * 16);
  const int64_t grid = (units + 7) / 8 * 8 * groups;
  if (grid > INT32_MAX) return BLAST_ERR_INVALID_ARG;
  d.n_units = (int)units;
  d.groups = (int)groups;
  using C = DecCfg<B, DUAL, NTT, XSMALL>;
  int64_t total = grid;
  if (plan.zero_job && plan.zero_job->hdr && !plan.zero_job->wide && plan.zero_job->max_chunks > 0 &&
      grid + plan.zero_job->max_chunks <= INT32_MAX) {
    ZeroJob& z = *plan.zero_job;
    d.main_blocks = (int)grid;
    d.z_blocks = (int)z.max_chunks;
    d.z_hdr = z.hdr;
    d.z_chunk_row = z.chunk_row;
    d.z_chunk_kb = z.chunk_kb;
    d.z_row_ptr = z.row_ptr;
    d.z_Y = z.Y;
    d.z_syt = z.syt;
    d.z_syi = z.syi;
    d.z_T = z.T;
    total = grid + z.max_chunks;
    z.done = true;
  }
  if constexpr (!DUAL && !CHUNK && !EPI::kOn) {
    if (a.act >= 0) {  // single matrix with an activation on the output
      static blast::DeviceFlags lds_set_post;
      if (int rc = ensure_lds_limit(reinterpret_cast<const void*>(&k_decode<B, false, NTT, false, XSMALL, true>),
                                    C::LDS_BYTES, lds_set_post))
        return rc;
      k_decode<B, false, NTT, false, XSMALL, true><<<dim3((unsigned)total), dim3(256), C::LDS_BYTES, stream>>>(d, epi);
      BLAST_LAUNCH_CHECK("k_decode");
      return BLAST_OK;
    }
  }
  static blast::DeviceFlags lds_set;
  if (int rc = ensure_lds_limit(reinterpret_cast<const void*>(&k_decode<B, DUAL, NTT, CHUNK, XSMALL, false, false, EPI>), C::LDS_BYTES,
                                lds_set))
    return rc;
  if constexpr (CHUNK) {
    if (!(plan.pre_zeroed && !plan.zeroed_wide)) {
      StreamArgs sa{a, 0, -1, 0, plan.hdr, plan.chunk_row, plan.chunk_kb, plan.chunk_ke};
      k_zero_shared_rows<B><<<dim3((unsigned)plan.max_chunks, (unsigned)((a.T + 63) / 64)), dim3(256), 0, stream>>>(sa);
      BLAST_LAUNCH_CHECK("k_zero_shared_rows");
    }
  }
  k_decode<B, DUAL, NTT, CHUNK, XSMALL, false, false, EPI><<<dim3((unsigned)total), dim3(256), C::LDS_BYTES, stream>>>(d, epi);
  BLAST_LAUNCH_CHECK("k_decode");
  return BLAST_OK;
}

template <int B, bool DUAL, class EPI>
int launch_decode(const TileArgs& a, const ChunkPlan& plan, hipStream_t stream, const EPI& epi) {
  if constexpr (!DUAL && !EPI::kOn) {
    // rows cut into chunks accumulate with fp32 atomics: only for fp32 output without an activation
    if (plan.hdr && !a.y_bf16 && a.act < 0) {
      if constexpr (B >= 64) {
        if (a.T <= 512 / B) return launch_decode_ntt<B, false, 1, true, 1>(a, plan, stream);
      }
      if constexpr (B == 128) {
        if (a.T <= 8) return launch_decode_ntt<B, false, 1, true, 2>(a, plan, stream);
      }
      if (a.T <= 16) return launch_decode_ntt<B, false, 1, true, 0>(a, plan, stream);
      return launch_decode_ntt<B, false, 2, true, 0>(a, plan, stream);
    }
  }
  ChunkPlan side{};  // no chunks; only the side job travels on
  side.zero_job = plan.zero_job;
  // the smallest activation tile that holds T token rows: 512 / B rows, at b = 128 also twice that
  if constexpr (B >= 64) {
    if (a.T <= 512 / B) return launch_decode_ntt<B, DUAL, 1, false, 1>(a, side, stream, epi);
  }
  if constexpr (B == 128) {
    if (a.T <= 8) return launch_decode_ntt<B, DUAL, 1, false, 2>(a, side, stream, epi);
  }
  if (a.T <= 16) return launch_decode_ntt<B, DUAL, 1, false, 0>(a, side, stream, epi);
  // groups of 32 tokens along gridDim.y (128-wide blocks: with a single activation tile per wave, see DecCfg)
  return launch_decode_ntt<B, DUAL, 2, false, 0>(a, side, stream, epi);
}

// Crossover with the streaming kernel, from token sweeps on the 1B-shaped MLP.  The decode kernel
// re-reads a matrix once per group of 16 or 32 tokens (from cache), the streaming kernel once per 256:
//  - up to 32 tokens the decode kernel always wins;
//  - the single-matrix product stays ahead up to 256 tokens as long as those re-reads are small
//    (the launch is latency bound; 13.8 us against 16.5 us at 256 tokens on a 3.3 MB matrix);
//  - the gated product (two matrices, twice the blocks per workgroup) crosses over at about 64 tokens,
//    unless its fullest block row is so long that the streaming kernel, which walks a whole row of the
//    gated product in one workgroup (the activation needs complete sums, so the row cannot be cut), would
//    spend longer on that one row than the decode kernel spends on everything (it deals a row's blocks to
//    the four waves of b/16 workgroups).  Measured on the 405B-class layer with the Zipf mask (fullest joint
//    row 256 blocks of 128 x 128): 183 us in the streaming kernel at 33-64 tokens, 0.7 us per block of that
//    row; the decode kernel takes about 42 us per group of 32 tokens there (174 MB of blocks per group):
//    84-93 us at 33-64 tokens, 120-127 us at 65-96, 168 us at 128.
constexpr int kDecodeAlwaysTokens = 32;
constexpr int kDecodeMaxTokens = 256;
constexpr int64_t kDecodeMaxRereadBytes = (int64_t)64 << 20;

template <bool DUAL>
bool decode_applies(int b, const TileArgs& a, int64_t nnz, int64_t max_row_blocks) {
  if (a.T <= kDecodeAlwaysTokens) return true;
  if (a.T > kDecodeMaxTokens) return false;
  const int64_t group = 32;  // tokens per unit of the decode kernel beyond 16 tokens
  const int64_t groups = (a.T + group - 1) / group;
  const int64_t reread = nnz * b * b * 2 * groups;
  if (DUAL) {
    // small products are a chain of latencies either way; the decode kernel's chain is the shorter one for up
    // to 64 tokens (1B / 3B shapes, b = 64: 17-19 us per MLP pass against 21-22 at 33-64 tokens; 8B shape,
    // b = 128: 25-28 against 29-32; from 96 tokens on the streaming kernel is ahead)
    if (groups <= 2 && reread <= kDecodeMaxRereadBytes) return true;
    if (max_row_blocks <= 0 || groups > 8) return false;
    const double row_us = (double)max_row_blocks * 0.7 * ((double)b * b / (128.0 * 128.0));  // streaming kernel, fullest row
    const double all_us = (double)reread / 4.1e6;                                            // decode kernel, whole product
    // only where that row is long against the fixed latencies of a launch (tens of microseconds)
    return row_us >= 30.0 && all_us < row_us;
  }
  return reread <= kDecodeMaxRereadBytes;
}

template <bool DUAL, class EPI = NoEpilogue>
int dispatch_tile(int b, const TileArgs& a, int64_t nnz, hipStream_t stream, const ChunkPlan& plan = ChunkPlan{},
                  bool ranged = false, const EPI& epi = EPI{}) {
  // the streaming kernel addresses activations with 32-bit byte offsets inside one column block
  const bool small_x = (int64_t)a.T * a.sxt * 2 < ((int64_t)1 << 32);
  const bool decode = a.x_vec && a.T > 0 && small_x && decode_applies<DUAL>(b, a, nnz, plan.max_row_blocks);
  if constexpr (!DUAL) {
    // (not where rows may be cut into chunks - fp32 output without an activation -, nor where this launch is to clear another
    // one's, nor for the last tokens of a longer call, whose rows are summed as the others')
    const bool chunks = plan.hdr && !a.y_bf16 && a.act < 0;
    if (a.x_vec && small_x && !ranged && !chunks && !plan.zero_job) {
      const int waves = a.T > kDecodeAlwaysTokens ? split_waves(b, a.nbr, a.T, nnz, plan.fullest, decode, cu_count()) : 0;
      if (waves == 4) return b == 64 ? launch_split<64, 4>(a, stream, epi) : launch_split<128, 4>(a, stream, epi);
      if (waves == 8) return b == 64 ? launch_split<64, 8>(a, stream, epi) : launch_split<128, 8>(a, stream, epi);
    }
  }
  if (decode) {
    // The decode kernel already spreads a block row over b/16 workgroups of four waves each, so a row of n
    // blocks is n/4 block steps deep.  Chunks (a zero-fill launch plus atomics, about 8 us on the 405B-class
    // gate matrix) only pay when that depth exceeds four times the average load of a workgroup slot
    // (measured there: fullest row 128 blocks, 20.8 us without chunks against 28.8 us with; 416 blocks, 42.0
    // against 23.3).
    ChunkPlan dplan = plan;
    if (dplan.hdr) {
      double ref = (double)nnz * (b / 16) / (4.0 * 2.0 * cu_count());
      if (ref < blast::kChunkBlocks) ref = blast::kChunkBlocks;
      if ((double)dplan.max_row_blocks / 4.0 <= 4.0 * ref) {
        dplan = ChunkPlan{};
        dplan.zero_job = plan.zero_job;
      }
    }
    switch (b) {
      case 32: return launch_decode<32, DUAL>(a, dplan, stream, epi);
      case 64: return launch_decode<64, DUAL>(a, dplan, stream, epi);
      case 128: return launch_decode<128, DUAL>(a, dplan, stream, epi);
      default: break;
    }
  }
  if (a.x_vec && a.T > 0 && !small_x && b >= 32) {
    // More tokens than 32-bit offsets reach: the same kernels over token ranges that each fit (whole
    // 256-token tiles, so no range ends inside a tile of the next one).
    const int64_t range = (((int64_t)1 << 32) - 1) / (a.sxt * 2) / 256 * 256;
    if (range >= 256) {
      for (int64_t t0 = 0; t0 < a.T; t0 += range) {
        TileArgs part = a;
        part.T = (int)((a.T - t0 < range) ? a.T - t0 : range);
        part.X = a.X + t0 * a.sxt;
        part.Y = static_cast<char*>(a.Y) + t0 * a.syt * (a.y_bf16 ? 2 : 4);
        if (int rc = dispatch_tile<DUAL>(b, part, nnz, stream, plan, true, epi.from(t0))) return rc;
      }
      return BLAST_OK;
    }
  }
  if (a.x_vec && a.T > 0 && small_x) {
    switch (b) {
      case 32: return launch_stream<32, DUAL>(a, plan, a.kdim, stream, epi);
      case 64: return launch_stream<64, DUAL>(a, plan, a.kdim, stream, epi);
      case 128: return launch_stream<128, DUAL>(a, plan, a.kdim, stream, epi);
      default: break;
    }
  }
  if (b == 16 && (a.x_vec || a.x_grp16) && a.T > 0) return launch_b16<DUAL>(a, nnz, stream, epi);
  switch (b) {
    case 16: return launch_tile<16, DUAL>(a, stream, epi);
    case 32: return launch_tile<32, DUAL>(a, stream, epi);
    case 64: return launch_tile<64, DUAL>(a, stream, epi);
    case 128: return launch_tile<128, DUAL>(a, stream, epi);
    default: return BLAST_ERR_UNSUPPORTED_BLOCK;
  }
}

int check_view(const blast_bsr_view* v) {
  if (!v) return BLAST_ERR_INVALID_ARG;
  if (v->rows < 0 || v->cols < 0 || v->nnz < 0) return BLAST_ERR_INVALID_ARG;
  if (!blast::supported_block(v->b)) return BLAST_ERR_UNSUPPORTED_BLOCK;
  if (v->rows % v->b || v->cols % v->b) return BLAST_ERR_SHAPE;
  if (v->rows / v->b > INT32_MAX / 2 || v->cols / v->b > INT32_MAX / 2 || v->nnz > INT32_MAX) return BLAST_ERR_INVALID_ARG;
  if (!v->row_ptr) return BLAST_ERR_INVALID_ARG;
  if (v->nnz > 0 && (!v->col_idx || !v->vals || !blast::aligned(v->vals, 16))) return BLAST_ERR_INVALID_ARG;
  return BLAST_OK;
}

int check_dense(const void* p, int64_t ld, int32_t layout, int64_t feat, int64_t T) {
  if (layout != BLAST_TOKEN_MAJOR && layout != BLAST_FEATURE_MAJOR) return BLAST_ERR_INVALID_ARG;
  if (T > 0 && feat > 0) {
    if (!p) return BLAST_ERR_INVALID_ARG;
    if (ld < (layout == BLAST_TOKEN_MAJOR ? feat : T)) return BLAST_ERR_INVALID_ARG;
  }
  return BLAST_OK;
}

void set_x(TileArgs& a, const uint16_t* X, int64_t ldx, int32_t layout) {
  a.X = X;
  if (layout == BLAST_TOKEN_MAJOR) {
    a.sxt = ldx;
    a.sxk = 1;
    a.x_vec = (ldx % 8 == 0 && blast::aligned(X, 16)) ? 1 : 0;
  } else {
    a.sxt = 1;
    a.sxk = ldx;
    a.x_vec = 0;
  }
}

void set_y(TileArgs& a, void* Y, int64_t ldy, int32_t layout, int32_t y_dtype) {
  a.Y = Y;
  a.y_bf16 = (y_dtype == BLAST_BF16) ? 1 : 0;
  a.y_fast = a.y_pairs = 0;
  if (layout == BLAST_TOKEN_MAJOR) {
    a.syt = ldy;
    a.syi = 1;
    a.y_fast = ((int64_t)256 * ldy * 4 + ldy * 4 < ((int64_t)1 << 31)) ? 1 : 0;
    a.y_pairs = (ldy % 2 == 0 && blast::aligned(Y, a.y_bf16 ? 4 : 8)) ? 1 : 0;
  } else {
    a.syt = 1;
    a.syi = ldy;
  }
}

MatDev mat_of(const blast_bsr_view* v) { return MatDev{v->row_ptr, v->col_idx, v->vals}; }

// The chunk plan costs a zero-fill launch and fp32 atomics on the split rows (measured: about 9 us on
// the 1B-shaped down projection, where it does not pay).  It is used only when the fullest block row,
// taken as one work item, would outlast four times the average load of a workgroup slot (and four
// chunks): then that row is the critical path of the launch by a wide margin.
ChunkPlan plan_of(const blast_bsr_view* v, int64_t T) {
  ChunkPlan p;
  p.fullest = v->max_row_blocks;
  if (!v->aux || v->max_row_blocks <= blast::kChunkBlocks) return p;
  const int64_t nbr = v->rows / v->b, nbc = v->cols / v->b;
  const int64_t tiles = (T + 255) / 256;
  double ref = (double)v->nnz * (double)tiles / (2.0 * cu_count());
  if (ref < blast::kChunkBlocks) ref = blast::kChunkBlocks;
  if ((double)v->max_row_blocks <= 4.0 * ref) return p;
  const blast::AuxLayout L = blast::aux_layout(nbr, nbc, v->nnz);
  const char* ab = static_cast<const char*>(v->aux);
  p.hdr = reinterpret_cast<const int*>(ab + L.hdr_off);
  p.chunk_row = reinterpret_cast<const int*>(ab + L.chunk_row_off);
  p.chunk_kb = reinterpret_cast<const int*>(ab + L.chunk_kb_off);
  p.chunk_ke = reinterpret_cast<const int*>(ab + L.chunk_ke_off);
  p.max_chunks = nbr + v->nnz / blast::kChunkBlocks;
  if (v->max_row_blocks > blast::kWideChunkBlocks) {  // otherwise every row is one wide chunk: no plan needed
    p.w_hdr = reinterpret_cast<const int*>(ab + L.whdr_off);
    p.w_chunk_row = reinterpret_cast<const int*>(ab + L.wchunk_row_off);
    p.w_chunk_kb = reinterpret_cast<const int*>(ab + L.wchunk_kb_off);
    p.w_chunk_ke = reinterpret_cast<const int*>(ab + L.wchunk_ke_off);
    p.w_max_chunks = nbr + v->nnz / blast::kWideChunkBlocks;
  }
  p.max_row_blocks = v->max_row_blocks;
  {
    // blocks per CU with 256-token tiles: below half a wide chunk, wide chunks are too coarse to balance
    const double per_cu = (double)v->nnz * (double)tiles / cu_count();
    p.stream_narrow = per_cu < blast::kWideChunkBlocks / 2;
  }
  return p;
}

}  // namespace
