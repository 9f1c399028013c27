// Products of scaled 8-bit operands (kern_linear8.h).
#include "scaled8_check.h"

#include "kern_linear8.h"

using namespace blast_dev;

namespace {

// Fewer 128-token tiles than this are cut into tiles of 32 whose blocks eight waves share, and up to 32 tokens any number.  Microseconds of
// 128-token tiles / of 32, bf16 results (8-bit ones within 4 %, fp32 ones 1 to 5 us more on both sides), with the number of the former.
// 64-wide, 2048 x 8192 at 90 %, 64 tiles 13.8 / 6.7, 192: 14.7 / 12.8, 256: 15.1 / 14.6, 288: 16.0 / 16.9; 6400 x 1600 at 80 %, 200: 9.0 /
// 7.8, 300: 9.3 / 10.6; 1600 x 6400 at 80 %, 225: 18.7 / 18.0, 250: 18.9 / 19.4; 8192 x 2048 at 50 %, 256, a tile to a CU: 16.2 / 14.7.
// Gated, 2048 x 8192, 128: 22.8 / 17.2, 192: 23.6 / 23.9; 6400 x 1600, 100: 13.3 / 10.7, 200: 14.0 / 19.4.  128-wide, 4096 x 14336 at 95 %,
// 128: 16.7 / 12.9, 192: 16.8 / 17.9, at 70 %, 128: 49 / 31, 192: 49 / 45, 224: 50 / 55; 14336 x 4096 at 95 %, 112: 9.8 / 7.8, 224: 10.7 /
// 13.9; gated 112: 16.7 / 16.7, at 70 % 38 / 32; 4096 x 14336, 128: 27.4 / 27.6, at 70 % 91 / 62.
template <int B, bool DUAL>
constexpr int64_t kFewTiles = B == 64 && !DUAL ? 256 : 144;

// Workgroups that have 32 rows of a block row each, where no scale needs all of them: up to 32 tokens, and where whole rows would be this
// many workgroups or fewer (us, 32 rows / whole; bf16; one token: 14336 x 4096 at 95 % 4.2 / 5.4, at 70 % 7.6 / 9.5, 4096 x 14336 at 95 %
// 4.2 / 6.5, 64-wide 8192 x 2048 at 90 % 3.7 / 4.1; 100 tokens: 4096 x 14336 at 95 %, 128 whole ones 6.9 / 7.2, at 70 % 17.9 / 16.8,
// 64-wide 2048 x 8192 at 90 % 5.2 / 5.6; 14336 x 4096 at 95 %, 448: 9.4 / 7.7, 64-wide 8192 x 2048, 512: 6.2 / 5.0).
constexpr int64_t kFewGroups = 128;

int check_weight(const blast_bsr_view* W, const blast_weight8_view* W8) {
  if (!W || !W->row_ptr || !W8 || !format8_ok(W8->format)) return BLAST_ERR_INVALID_ARG;
  if (W->rows < 0 || W->cols < 0 || W->nnz < 0 || W->nnz > INT32_MAX) return BLAST_ERR_INVALID_ARG;
  if (W->b != 64 && W->b != 128) return BLAST_ERR_UNSUPPORTED_BLOCK;
  if (W->rows % W->b || W->cols % W->b) return BLAST_ERR_SHAPE;
  if (W->rows > INT32_MAX / 2 || W->cols > INT32_MAX / 2) return BLAST_ERR_INVALID_ARG;
  if (W->nnz > 0 && (!W->col_idx || !W8->vals8 || !blast::aligned(W8->vals8, 16) || !W8->scales || !blast::aligned(W8->scales, 16)))
    return BLAST_ERR_INVALID_ARG;
  return BLAST_OK;
}

Mat8 mat8_of(const blast_bsr_view* W, const blast_weight8_view* W8) { return Mat8{W->row_ptr, W->col_idx, W8->vals8, W8->scales}; }

// An output in scaled 8-bit form: in groups of a block's rows.
int check_out8(const blast_scaled8_view* v, const blast_bsr_view* W, int64_t T) {
  if (!v) return BLAST_OK;
  if (v->group != W->b) return BLAST_ERR_INVALID_ARG;
  return check_eight(v, T, W->rows, 16);
}

int cu_count8() {
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 256;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) return 256;
  return n;
}

// Workgroups for tiles of TT tokens: one for each, or as many as are resident at once; 0: more tiles than can be counted.  Many tiles: two
// XCDs share a block row, each with half of its tokens (us, one / two / four / eight XCDs to a row: 53248 x 16384 at 95 %, 2048 tokens 191
// / 189 / 191 / 192; gated 14336 x 4096, 4096 tokens 99 / 100 / 100 / 99; 2048 x 8192 at 90 %, 64-wide, 2048 tokens 24.0 / 22.8 / 22.2 /
// 22.0).  An odd number of tiles leaves one of two XCDs a tile short.
int64_t grid8(Linear8Args& a, int TT, int64_t resident) {
  a.ntt = (int)(((int64_t)a.T + TT - 1) / TT);
  a.parts = TT >= 128 && a.ntt >= 2 && (a.ntt % 2 == 0 || a.ntt >= 16) ? 2 : 1;
  const int64_t rows = 8 / a.parts;
  const int64_t most = (((int64_t)a.nbr + rows - 1) / rows) * (((int64_t)a.ntt + a.parts - 1) / a.parts);  // of an XCD
  if (most > INT32_MAX / 8) return 0;
  return 8 * (most < resident / 8 ? most : resident / 8 < 1 ? 1 : resident / 8);
}

template <class K>
int raise_lds(K kernel, int bytes, blast::DeviceFlags& set) {
  int dev = 0;
  BLAST_HIP_TRY(hipGetDevice(&dev));
  if (!set.test(dev)) {
    BLAST_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    set.set(dev);
  }
  return BLAST_OK;
}

template <int B, int ROWS, bool DUAL, int WF, int XF>
int launch_split(Linear8Args a, hipStream_t stream) {
  using C = S8Cfg<B, ROWS, DUAL>;
  static blast::DeviceFlags set;
  if (int rc = raise_lds(&k_linear8_split<B, ROWS, DUAL, WF, XF>, C::LDS_BYTES, set)) return rc;
  const int64_t grid = grid8(a, C::TT, INT32_MAX);
  if (grid == 0) return BLAST_ERR_INVALID_ARG;
  k_linear8_split<B, ROWS, DUAL, WF, XF><<<dim3((unsigned)grid, B / ROWS), dim3(64 * C::NW), C::LDS_BYTES, stream>>>(a);
  BLAST_LAUNCH_CHECK("k_linear8_split");
  return BLAST_OK;
}

template <int B, bool DUAL, int WF, int XF>
int launch_linear8(Linear8Args a, hipStream_t stream) {
  const int64_t tiles = (int64_t)a.nbr * (((int64_t)a.T + 127) / 128);
  static blast::DeviceFlags tile_set;
  // (a workgroup of 512 lanes to a block row and 32 tokens: not more than a launch has lanes for; lists have any number)
  const bool few = a.T <= 32 && a.nbr < blast::most_groups(512);
  if (few || tiles < kFewTiles<B, DUAL>) {
    if (a.y8.codes || a.k8[0].codes || a.k8[1].codes) return launch_split<B, B, DUAL, WF, XF>(a, stream);
    const int64_t groups = (int64_t)a.nbr * (((int64_t)a.T + 31) / 32);
    if (a.T <= 32 || groups <= kFewGroups) return launch_split<B, 32, DUAL, WF, XF>(a, stream);
    return launch_split<B, B, DUAL, WF, XF>(a, stream);
  }
  using C = L8Cfg<B>;
  if (int rc = raise_lds(&k_linear8<B, DUAL, WF, XF>, C::LDS_BYTES, tile_set)) return rc;
  const int64_t grid = grid8(a, C::TT, 2 * cu_count8());
  if (grid == 0) return BLAST_ERR_INVALID_ARG;
  k_linear8<B, DUAL, WF, XF><<<dim3((unsigned)grid), dim3(256), C::LDS_BYTES, stream>>>(a);
  BLAST_LAUNCH_CHECK("k_linear8");
  return BLAST_OK;
}

template <int B, bool DUAL>
int by_formats(const Linear8Args& a, hipStream_t stream) {
  if (a.wfmt == BLAST_E4M3)
    return a.x.fmt == BLAST_E4M3 ? launch_linear8<B, DUAL, 0, 0>(a, stream) : launch_linear8<B, DUAL, 0, 1>(a, stream);
  return a.x.fmt == BLAST_E4M3 ? launch_linear8<B, DUAL, 1, 0>(a, stream) : launch_linear8<B, DUAL, 1, 1>(a, stream);
}

}  // namespace

extern "C" int blast_bsr_linear_scaled8(const blast_bsr_view* W, const blast_weight8_view* W8, const blast_scaled8_view* X, int64_t T,
                                        const float* bias, int32_t act, const void* R, int64_t ldr, int32_t r_dtype, void* Y,
                                        int64_t ldy, int32_t y_dtype, const blast_scaled8_view* Y8, const blast_scaled8_view* Z8,
                                        void* stream_) {
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (int rc = check_weight(W, W8)) return rc;
  if (T < 0 || T > INT32_MAX / 2) return BLAST_ERR_INVALID_ARG;
  if (act < BLAST_ACT_NONE || act > BLAST_ACT_RELU) return BLAST_ERR_INVALID_ARG;
  if (Y && y_dtype != BLAST_F32 && y_dtype != BLAST_BF16) return BLAST_ERR_INVALID_ARG;
  if (R && r_dtype != BLAST_F32 && r_dtype != BLAST_BF16) return BLAST_ERR_INVALID_ARG;
  if (int rc = check_eight(X, T, W->cols, 16)) return rc;
  if (X->group < W->b) return BLAST_ERR_INVALID_ARG;
  if (int rc = check_out8(Y8, W, T)) return rc;
  if (int rc = check_out8(Z8, W, T)) return rc;
  if (T == 0 || W->rows == 0) return BLAST_OK;
  if (!Y && !Y8) return BLAST_ERR_INVALID_ARG;
  if ((Y && ldy < W->rows) || (R && ldr < W->rows)) return BLAST_ERR_INVALID_ARG;
  if (W->cols == 0 && W->nnz > 0) return BLAST_ERR_SHAPE;
  Linear8Args a{};
  a.m[0] = mat8_of(W, W8);
  a.row_order = W->row_order;
  a.x = eight_of(X);
  a.wfmt = W8->format;
  a.T = (int)T;
  a.nbr = (int)(W->rows / W->b);
  a.act = act;
  a.bias = bias;
  a.r = R;
  a.ldr = ldr;
  a.r_bf16 = r_dtype == BLAST_BF16;
  a.y = Y;
  a.ldy = ldy;
  a.y_bf16 = y_dtype == BLAST_BF16;
  a.r_vec = blast::aligned(R, 16) && ldr * (a.r_bf16 ? 2 : 4) % 16 == 0;
  a.y_vec = blast::aligned(Y, 16) && ldy * (a.y_bf16 ? 2 : 4) % 16 == 0;
  if (Y8) a.y8 = eight_of(Y8);
  if (Z8) a.k8[0] = eight_of(Z8);
  return W->b == 64 ? by_formats<64, false>(a, stream) : by_formats<128, false>(a, stream);
}

extern "C" int blast_bsr_gated_scaled8(const blast_bsr_view* Wgate, const blast_weight8_view* gate8, const blast_bsr_view* Wup,
                                       const blast_weight8_view* up8, const blast_scaled8_view* X, int64_t T, int32_t act, uint16_t* H,
                                       int64_t ldh, const blast_scaled8_view* H8, const blast_scaled8_view* G8,
                                       const blast_scaled8_view* U8, void* stream_) {
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (int rc = check_weight(Wgate, gate8)) return rc;
  if (int rc = check_weight(Wup, up8)) return rc;
  if (Wgate->rows != Wup->rows || Wgate->cols != Wup->cols || Wgate->b != Wup->b) return BLAST_ERR_SHAPE;
  if (gate8->format != up8->format) return BLAST_ERR_INVALID_ARG;
  if (T < 0 || T > INT32_MAX / 2) return BLAST_ERR_INVALID_ARG;
  if (act < BLAST_ACT_NONE || act > BLAST_ACT_RELU) return BLAST_ERR_INVALID_ARG;
  if (int rc = check_eight(X, T, Wgate->cols, 16)) return rc;
  if (X->group < Wgate->b) return BLAST_ERR_INVALID_ARG;
  const blast_scaled8_view* outs[] = {H8, G8, U8};
  for (const blast_scaled8_view* o : outs)
    if (int rc = check_out8(o, Wgate, T)) return rc;
  if (T == 0 || Wgate->rows == 0) return BLAST_OK;
  if ((H != nullptr) == (H8 != nullptr)) return BLAST_ERR_INVALID_ARG;
  if (H && ldh < Wgate->rows) return BLAST_ERR_INVALID_ARG;
  if (Wgate->cols == 0 && (Wgate->nnz > 0 || Wup->nnz > 0)) return BLAST_ERR_SHAPE;
  Linear8Args a{};
  a.m[0] = mat8_of(Wgate, gate8);
  a.m[1] = mat8_of(Wup, up8);
  a.row_order = Wgate->row_order;
  a.x = eight_of(X);
  a.wfmt = gate8->format;
  a.T = (int)T;
  a.nbr = (int)(Wgate->rows / Wgate->b);
  a.act = act;
  a.y = H;
  a.ldy = ldh;
  a.y_bf16 = 1;
  a.y_vec = blast::aligned(H, 16) && ldh * 2 % 16 == 0;
  if (H8) a.y8 = eight_of(H8);
  if (G8) a.k8[0] = eight_of(G8);
  if (U8) a.k8[1] = eight_of(U8);
  return Wgate->b == 64 ? by_formats<64, true>(a, stream) : by_formats<128, true>(a, stream);
}
