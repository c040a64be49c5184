// Matrix products of ragged groups of rows: C[r] = B_g A[r], its transpose, and the sum of the outer products of a group.
#include "layers.h"

namespace adacgd {
namespace {

constexpr int kTileShift = 6, kTileRows = 1 << kTileShift;

struct ProductArgs {
  const void* a;
  const void* b;
  void* c;
  const int64_t* offsets;
  int64_t rows, groups, each;           // `each` entries of offsets to a group
  int64_t lda, ldb, ldc, gsb, gsc;
  int n, k;
};

// C tile of 64 x 64 from A(m, r) and B(n, r) summed over r, any layout: element (m, r) of A is at m am + r ar.
template <typename T, typename O>
__device__ void tile_product(const T* a, int64_t am, int64_t ar, int m, const T* b, int64_t bn, int64_t br, int n, int64_t red,
                             O* c, int64_t cm) {
  __shared__ float As[16][64 + 1], Bs[16][64 + 1];
  const int t = threadIdx.x, tx = t % 16, ty = t / 16;
  float acc[4][4] = {};
  for (int64_t r0 = 0; r0 < red; r0 += 16) {
    for (int i = t; i < 16 * 64; i += 256) {
      const int r = i % 16, q = i / 16;
      const bool in = r0 + r < red;
      As[r][q] = in && q < m ? to_float(a[q * am + (r0 + r) * ar]) : 0.f;
      Bs[r][q] = in && q < n ? to_float(b[q * bn + (r0 + r) * br]) : 0.f;
    }
    __syncthreads();
    for (int r = 0; r < 16; ++r)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(As[r][ty * 4 + i], Bs[r][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j)
      if (ty * 4 + i < m && tx * 4 + j < n) c[(ty * 4 + i) * cm + tx * 4 + j] = from_float<O>(acc[i][j]);
}

template <typename T, typename O, bool TRANSPOSED>
__global__ void __launch_bounds__(256) k_rows_product(ProductArgs p) {
  const Slice s = find_slice(p.offsets, p.groups, p.rows, p.each, kTileShift, blockIdx.y);
  if (s.group < 0 || s.end <= s.begin) return;
  const int cols = TRANSPOSED ? p.k : p.n, red = TRANSPOSED ? p.n : p.k;
  const int c0 = blockIdx.x * 64;
  const T* b = (const T*)p.b + s.group * p.gsb;
  tile_product<T, O>((const T*)p.a + s.begin * p.lda, p.lda, 1, (int)(s.end - s.begin), TRANSPOSED ? b + c0 : b + c0 * p.ldb,
                     TRANSPOSED ? 1 : p.ldb, TRANSPOSED ? p.ldb : 1, cols - c0, red, (O*)p.c + s.begin * p.ldc + c0, p.ldc);
}

template <typename T, typename O>
__global__ void __launch_bounds__(256) k_group_product(ProductArgs p) {
  const int64_t g = blockIdx.z;
  const int64_t first = offset_at(p.offsets, g, p.rows);
  int64_t last = offset_at(p.offsets, g + 1, p.rows);
  if (last < first) last = first;
  const int n0 = blockIdx.y * 64, k0 = blockIdx.x * 64;
  tile_product<T, O>((const T*)p.a + first * p.lda + n0, 1, p.lda, p.n - n0, (const T*)p.b + first * p.ldb + k0, 1, p.ldb, p.k - k0,
                     last - first, (O*)p.c + g * p.gsc + n0 * p.ldc + k0, p.ldc);
}

int check_sizes(int32_t product, int64_t rows, int64_t groups, int64_t n, int64_t k) {
  if (product < ADACGD_FORWARD || product > ADACGD_DW) return fail(ADACGD_ERR_ARG, "unknown product %d", product);
  ADACGD_TRY(check_count("rows", rows, 0, kMaxCount));
  ADACGD_TRY(check_count("groups", groups, 1, 65535));
  ADACGD_TRY(check_count("n", n, 1, kMaxColumns));
  ADACGD_TRY(check_count("k", k, 1, kMaxColumns));
  return ADACGD_OK;
}

template <typename T, typename O>
int launch(int32_t product, const ProductArgs& p, hipStream_t stream) {
  if (product == ADACGD_DW) {
    k_group_product<T, O><<<dim3((p.k + 63) / 64, (p.n + 63) / 64, p.groups), 256, 0, stream>>>(p);
  } else {
    const int64_t slices = slice_numbers(p.rows, p.groups, kTileShift);
    if (product == ADACGD_FORWARD) k_rows_product<T, O, false><<<dim3((p.n + 63) / 64, slices), 256, 0, stream>>>(p);
    else k_rows_product<T, O, true><<<dim3((p.k + 63) / 64, slices), 256, 0, stream>>>(p);
  }
  return launched("adacgd_group_matmul");
}

}  // namespace
}  // namespace adacgd

using namespace adacgd;

extern "C" {

int adacgd_group_matmul_workspace_bytes(int32_t product, int32_t dtype, int64_t rows, int64_t groups, int64_t n, int64_t k, int64_t* bytes) {
  if (!bytes) return fail(ADACGD_ERR_ARG, "bytes is null");
  if (dtype < 0 || dtype > ADACGD_FP16) return fail(ADACGD_ERR_ARG, "unknown type %d", dtype);
  ADACGD_TRY(check_sizes(product, rows, groups, n, k));
  *bytes = 0;
  return ADACGD_OK;
}

int adacgd_group_matmul(int32_t product, int64_t rows, int64_t groups, int64_t n, int64_t k, const int64_t* offsets,
                        const adacgd_tensor* a, const adacgd_tensor* b, const adacgd_tensor* c, void* workspace,
                        int64_t workspace_bytes, void* stream) {
  ADACGD_TRY(check_sizes(product, rows, groups, n, k));
  if (!offsets) return fail(ADACGD_ERR_ARG, "offsets is null");
  const bool dw = product == ADACGD_DW;
  ADACGD_TRY(check_tensor(a, "a", rows, product == ADACGD_FORWARD ? k : n, false, false));
  ADACGD_TRY(check_tensor(b, "b", dw ? rows : n, k, !dw, true));
  ADACGD_TRY(check_tensor(c, "c", dw ? n : rows, product == ADACGD_FORWARD ? n : k, dw && groups > 1, false));
  if (a->dtype != b->dtype) return fail(ADACGD_ERR_ARG, "a and b differ in type");
  if (c->dtype != a->dtype && c->dtype != ADACGD_FP32) return fail(ADACGD_ERR_ARG, "c has neither the type of a and b nor fp32");
  int64_t need = 0;
  ADACGD_TRY(adacgd_group_matmul_workspace_bytes(product, a->dtype, rows, groups, n, k, &need));
  ADACGD_TRY(check_workspace(workspace, workspace_bytes, need));
  if (rows == 0 && !dw) return ADACGD_OK;
  ProductArgs p{a->data, b->data, c->data, offsets, rows, groups, 1, a->stride, b->stride, c->stride, b->group_stride, c->group_stride, (int)n, (int)k};
  if (!dw && b->group_stride == 0) { p.each = groups; p.groups = 1; }      // one matrix for all: one group
  return by_dtype(a->dtype, [&](auto t) {
    using T = decltype(t);
    if (c->dtype == ADACGD_FP32) return launch<T, float>(product, p, (hipStream_t)stream);
    return launch<T, T>(product, p, (hipStream_t)stream);
  });
}

}  // extern "C"
