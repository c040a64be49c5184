// Layer normalisation, its gradients by group of rows, and dropout from the counter-based generator.
#include <cmath>

#include "layers.h"
#include "quant.h"

namespace adacgd {
namespace {

__device__ __forceinline__ float block_sum(float v, float* lds) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if (lane_id() == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) s += lds[w];
  return s;
}

template <typename T>
__global__ void __launch_bounds__(256) k_norm(const T* x, int64_t ldx, const float* weight, const float* bias, int d, float eps, T* y, int64_t ldy, float* mean, float* rstd) {
  __shared__ float lds[4];
  const int64_t row = blockIdx.x;
  x += row * ldx;
  y += row * ldy;
  float s = 0.f;
  for (int c = threadIdx.x; c < d; c += 256) s += to_float(x[c]);
  const float m = block_sum(s, lds) / d;
  s = 0.f;
  for (int c = threadIdx.x; c < d; c += 256) { const float v = to_float(x[c]) - m; s += v * v; }
  const float r = 1.f / sqrtf(block_sum(s, lds) / d + eps);
  for (int c = threadIdx.x; c < d; c += 256) {
    const float h = (to_float(x[c]) - m) * r;
    y[c] = from_float<T>(h * (weight ? weight[c] : 1.f) + (bias ? bias[c] : 0.f));
  }
  if (threadIdx.x == 0 && mean) { mean[row] = m; rstd[row] = r; }
}

template <typename T>
__global__ void __launch_bounds__(256) k_norm_dx(const int64_t* offsets, int64_t groups, int64_t rows, const T* dy, int64_t ldy, const T* x, int64_t ldx, const float* weight, const float* mean, const float* rstd, int d, T* dx, int64_t ldd) {
  __shared__ float lds[4];
  const int64_t row = blockIdx.x;
  if (row < offset_at(offsets, 0, rows) || row >= offset_at(offsets, groups, rows)) return;
  x += row * ldx; dy += row * ldy; dx += row * ldd;
  const float m = mean[row], r = rstd[row];
  float s = 0.f, q = 0.f;
  for (int c = threadIdx.x; c < d; c += 256) {
    const float g = to_float(dy[c]) * (weight ? weight[c] : 1.f);
    s += g;
    q += g * ((to_float(x[c]) - m) * r);
  }
  s = block_sum(s, lds) / d;
  q = block_sum(q, lds) / d;
  for (int c = threadIdx.x; c < d; c += 256) {
    const float g = to_float(dy[c]) * (weight ? weight[c] : 1.f);
    dx[c] = from_float<T>(r * (g - s - (to_float(x[c]) - m) * r * q));
  }
}

template <typename T>
__global__ void __launch_bounds__(64) k_norm_dw(const int64_t* offsets, int64_t rows, const T* dy, int64_t ldy, const T* x, int64_t ldx, const float* mean, const float* rstd, int d, float* dw, int64_t ldw, float* db, int64_t ldb) {
  const int64_t g = blockIdx.y;
  const int c = blockIdx.x * 64 + threadIdx.x;
  const int64_t first = offset_at(offsets, g, rows), last = offset_at(offsets, g + 1, rows);
  if (c >= d) return;
  float sw = 0.f, sb = 0.f;
  for (int64_t row = first; row < last; ++row) {
    const float v = to_float(dy[row * ldy + c]);
    sw += v * ((to_float(x[row * ldx + c]) - mean[row]) * rstd[row]);
    sb += v;
  }
  if (dw) dw[g * ldw + c] = sw;
  if (db) db[g * ldb + c] = sb;
}

template <typename T>
__global__ void __launch_bounds__(256) k_dropout(const T* x, int64_t ldx, const T* residual, int64_t ldr, T* out, int64_t ldo, int64_t rows, int d, uint32_t cut, float scale, uint64_t seed, uint32_t step, const int64_t* step_dev, uint32_t layer, uint64_t first) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows * d) return;
  const int64_t r = i / d, c = i % d;
  const uint64_t e = first + (uint64_t)i;
  if (step_dev) step += (uint32_t)*step_dev;
  uint32_t w[4];
  philox4x32_10((uint32_t)(e >> 3), (uint32_t)(e >> 35), step, layer + 1, (uint32_t)seed, (uint32_t)(seed >> 32), w);
  const uint32_t h = e & 7;
  const uint32_t word = h < 4 ? (h < 2 ? w[0] : w[1]) : (h < 6 ? w[2] : w[3]);
  const uint32_t draw = h & 1 ? word >> 16 : word & 0xffff;
  float v = draw >= cut ? to_float(x[r * ldx + c]) * scale : 0.f;
  if (residual) v += to_float(residual[r * ldr + c]);
  out[r * ldo + c] = from_float<T>(v);
}

}  // namespace
}  // namespace adacgd

using namespace adacgd;

extern "C" {

int adacgd_layer_norm(int64_t rows, int64_t d, const adacgd_tensor* x, const float* weight, const float* bias, double eps,
                      const adacgd_tensor* y, float* mean, float* rstd, void* stream) {
  ADACGD_TRY(check_count("rows", rows, 0, kMaxCount));
  ADACGD_TRY(check_count("d", d, 1, kMaxColumns));
  ADACGD_TRY(check_tensor(x, "x", rows, d, false, false));
  ADACGD_TRY(check_tensor(y, "y", rows, d, false, false));
  if (x->dtype != y->dtype) return fail(ADACGD_ERR_ARG, "x and y differ in type");
  if (!std::isfinite(eps) || eps < 0) return fail(ADACGD_ERR_ARG, "eps must be finite and >= 0");
  if (!mean != !rstd) return fail(ADACGD_ERR_ARG, "mean and rstd are given together or not at all");
  if (rows == 0) return ADACGD_OK;
  return by_dtype(x->dtype, [&](auto t) {
    using T = decltype(t);
    k_norm<T><<<rows, 256, 0, (hipStream_t)stream>>>((const T*)x->data, x->stride, weight, bias, (int)d, (float)eps, (T*)y->data, y->stride, mean, rstd);
    return launched("adacgd_layer_norm");
  });
}

int adacgd_layer_norm_backward_workspace_bytes(int64_t rows, int64_t groups, int64_t d, int64_t* bytes) {
  if (!bytes) return fail(ADACGD_ERR_ARG, "bytes is null");
  ADACGD_TRY(check_count("rows", rows, 0, kMaxCount));
  ADACGD_TRY(check_count("groups", groups, 1, 65535));
  ADACGD_TRY(check_count("d", d, 1, kMaxColumns));
  *bytes = 0;
  return ADACGD_OK;
}

int adacgd_layer_norm_backward(int64_t rows, int64_t groups, int64_t d, const int64_t* offsets, const adacgd_tensor* dy,
                               const adacgd_tensor* x, const float* weight, const float* mean, const float* rstd,
                               const adacgd_tensor* dx, const adacgd_tensor* dweight, const adacgd_tensor* dbias,
                               void* workspace, int64_t workspace_bytes, void* stream) {
  int64_t need = 0;
  ADACGD_TRY(adacgd_layer_norm_backward_workspace_bytes(rows, groups, d, &need));
  if (!offsets) return fail(ADACGD_ERR_ARG, "offsets is null");
  ADACGD_TRY(check_tensor(dy, "dy", rows, d, false, false));
  ADACGD_TRY(check_tensor(x, "x", rows, d, false, false));
  ADACGD_TRY(check_tensor(dx, "dx", rows, d, false, false));
  if (x->dtype != dy->dtype || x->dtype != dx->dtype) return fail(ADACGD_ERR_ARG, "dy, x and dx differ in type");
  if (rows > 0 && (!mean || !rstd)) return fail(ADACGD_ERR_ARG, "mean or rstd is null");
  for (const adacgd_tensor* t : {dweight, dbias}) {
    if (!t) continue;
    const char* name = t == dweight ? "dweight" : "dbias";
    ADACGD_TRY(check_tensor(t, name, groups, d, false, false));
    if (t->dtype != ADACGD_FP32) return fail(ADACGD_ERR_ARG, "%s must be fp32", name);
  }
  ADACGD_TRY(check_workspace(workspace, workspace_bytes, need));
  return by_dtype(x->dtype, [&](auto t) -> int {
    using T = decltype(t);
    if (rows > 0) {
      k_norm_dx<T><<<rows, 256, 0, (hipStream_t)stream>>>(offsets, groups, rows, (const T*)dy->data, dy->stride, (const T*)x->data, x->stride, weight, mean, rstd, (int)d, (T*)dx->data, dx->stride);
      ADACGD_TRY(launched("adacgd_layer_norm_backward"));
    }
    if (dweight || dbias)
      k_norm_dw<T><<<dim3((d + 63) / 64, groups), 64, 0, (hipStream_t)stream>>>(offsets, rows, (const T*)dy->data, dy->stride, (const T*)x->data, x->stride, mean, rstd, (int)d,
                                                                     dweight ? (float*)dweight->data : nullptr, dweight ? dweight->stride : 0, dbias ? (float*)dbias->data : nullptr, dbias ? dbias->stride : 0);
    return launched("adacgd_layer_norm_backward");
  });
}

int adacgd_dropout(int64_t rows, int64_t d, const adacgd_tensor* x, const adacgd_tensor* residual, const adacgd_tensor* out,
                   double p, uint64_t seed, uint32_t step, const int64_t* step_dev, uint32_t layer, uint64_t first, void* stream) {
  ADACGD_TRY(check_count("rows", rows, 0, kMaxCount));
  ADACGD_TRY(check_count("d", d, 1, kMaxColumns));
  ADACGD_TRY(check_tensor(x, "x", rows, d, false, false));
  if (residual) ADACGD_TRY(check_tensor(residual, "residual", rows, d, false, false));
  ADACGD_TRY(check_tensor(out, "out", rows, d, false, false));
  if (x->dtype != out->dtype || (residual && residual->dtype != x->dtype)) return fail(ADACGD_ERR_ARG, "x, residual and out differ in type");
  if (!(p >= 0 && p <= 1)) return fail(ADACGD_ERR_ARG, "p must be in [0, 1]");
  if (layer == 0xffffffffu) return fail(ADACGD_ERR_ARG, "layer must be below 2^32 - 1");
  if (rows == 0) return ADACGD_OK;
  const uint32_t cut = (uint32_t)std::floor(p * 65536 + 0.5);
  const float scale = cut == 65536 ? 0.f : (float)(65536.0 / (65536 - cut));
  return by_dtype(x->dtype, [&](auto t) {
    using T = decltype(t);
    k_dropout<T><<<(rows * d + 255) / 256, 256, 0, (hipStream_t)stream>>>((const T*)x->data, x->stride, residual ? (const T*)residual->data : nullptr, residual ? residual->stride : 0,
                                                               (T*)out->data, out->stride, rows, (int)d, cut, scale, seed, step, step_dev, layer, first);
    return launched("adacgd_dropout");
  });
}

}  // extern "C"
