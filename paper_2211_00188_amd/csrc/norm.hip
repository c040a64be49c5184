// Layer normalisation, its gradients by group of rows, and dropout from the counter-based generator.
#include <cmath>
#include <type_traits>

#include "layers.h"
#include "quant.h"

namespace adacgd {
namespace {

// A row is held in registers: `TPR` threads, `NV` vectors of 16 bytes each, vector i of thread t being number i TPR + t of the
// row, so that x is read once whatever is made of it.  One wavefront to a row needs no barrier; rows past what 1024 threads
// hold are read again (they are in cache).  The least threads that hold the row are taken, with one or two vectors each: four need
// the registers that rows on their way ahead take (65536 x 2048 bf16 forward: 168 us by a wavefront to a row, 116 by 256 threads).  Short
// rows share a wavefront: 10^6 of 64 elements 66 us forward (289 by a wavefront each), 3 10^5 of 256 elements 62 us forward and 109
// backward (87 and 215).  Bound by memory: a pass over x and one over y, or over dy, x and dx; 65536 x 2048 bf16 116 us forward
// (4.6 TB/s) and 190 backward (4.2), fp32 213 and 327 (5.0 and 4.9).
template <int TPR, int BLOCK>
__device__ __forceinline__ float row_sum(float v, float* lds) {
  if constexpr (TPR == 16) return row16_sumf(v);
  v = wave_sumf(v);
  if constexpr (TPR == 64) return v;
  __syncthreads();
  if (lane_id() == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < BLOCK / 64; ++w) s += lds[w];
  return s;
}
// Two sums at once.
template <int TPR, int BLOCK>
__device__ __forceinline__ void row_sums(float& a, float& b, float* lds) {
  if constexpr (TPR == 16) {
    a = row16_sumf(a);
    b = row16_sumf(b);
    return;
  }
  a = wave_sumf(a);
  b = wave_sumf(b);
  if constexpr (TPR == 64) return;
  __syncthreads();
  if (lane_id() == 0) { lds[threadIdx.x / 64] = a; lds[16 + threadIdx.x / 64] = b; }
  __syncthreads();
  a = b = 0.f;
#pragma unroll
  for (int w = 0; w < BLOCK / 64; ++w) { a += lds[w]; b += lds[16 + w]; }
}

// Elements of weight or bias that belong to a thread's vectors.
template <int NV, int E, int TPR>
__device__ __forceinline__ void load_columns(const float* p, float missing, int t, int d, float (&o)[NV][E]) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + t) * E;
#pragma unroll
    for (int j = 0; j < E; ++j) o[i][j] = p && c + j < d ? p[c + j] : missing;
  }
}

template <typename T, int TPR, int NV, int BLOCK>
__global__ void __launch_bounds__(BLOCK) k_norm(const T* x, int64_t ldx, const float* weight, const float* bias, int64_t rows, int d, float eps,
                                                T* y, int64_t ldy, float* mean, float* rstd) {
  constexpr int E = Vec<T>::kElems, PER = BLOCK / TPR;
  __shared__ float lds[32];
  const int t = threadIdx.x % TPR;
  float w[NV][E], b[NV][E];
  load_columns<NV, E, TPR>(weight, 1.f, t, d, w);
  load_columns<NV, E, TPR>(bias, 0.f, t, d, b);
  Vec<T> next[NV];
  const auto load = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < NV; ++i) next[i].load(x + row * ldx + (i * TPR + t) * E, d - (i * TPR + t) * E);
  };
  int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / TPR;
  const int64_t step = (int64_t)gridDim.x * PER;
  if (row < rows) load(row);
  for (; row < rows; row += step) {
    Vec<T> v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = next[i];
    if (row + step < rows) load(row + step);             // (on its way while this row is worked on)
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < E; ++j) s += v[i].get(j);
    const float m = row_sum<TPR, BLOCK>(s, lds) / d;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const float c = (i * TPR + t) * E + j < d ? v[i].get(j) - m : 0.f;
        s = fmaf(c, c, s);
      }
    const float r = 1.f / sqrtf(row_sum<TPR, BLOCK>(s, lds) / d + eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float f[E];
#pragma unroll
      for (int j = 0; j < E; ++j) f[j] = fmaf((v[i].get(j) - m) * r, w[i][j], b[i][j]);
      Vec<T> o;
      o.put(f);
      o.store(y + row * ldy + (i * TPR + t) * E, d - (i * TPR + t) * E);
    }
    if (t == 0 && mean) { mean[row] = m; rstd[row] = r; }
  }
}

// Rows longer than registers hold, in three passes over the row: 16384 x 12288 fp32 643 us forward (2.5 TB/s of x and y once).
template <typename T>
__global__ void __launch_bounds__(1024) k_norm_long(const T* x, int64_t ldx, const float* weight, const float* bias, int64_t rows, int d, float eps,
                                                    T* y, int64_t ldy, float* mean, float* rstd) {
  __shared__ float lds[32];
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const T* xr = x + row * ldx;
    T* yr = y + row * ldy;
    float s = 0.f;
    for (int c = threadIdx.x; c < d; c += 1024) s += to_float(xr[c]);
    const float m = row_sum<1024, 1024>(s, lds) / d;
    s = 0.f;
    for (int c = threadIdx.x; c < d; c += 1024) { const float v = to_float(xr[c]) - m; s += v * v; }
    const float r = 1.f / sqrtf(row_sum<1024, 1024>(s, lds) / d + eps);
    for (int c = threadIdx.x; c < d; c += 1024) yr[c] = from_float<T>((to_float(xr[c]) - m) * r * (weight ? weight[c] : 1.f) + (bias ? bias[c] : 0.f));
    if (threadIdx.x == 0 && mean) { mean[row] = m; rstd[row] = r; }
  }
}

// Where the gradients of weight and bias go: the output of a group that is one slice, else the slice's own partial sums.
struct Columns {
  float* dw;
  float* db;
  int64_t ldw, ldb;
  float* partial;       // [numbers of slices][2][d]
  int shift;
};
__device__ __forceinline__ void places(const Columns& out, const Slice& s, int64_t number, int d, float*& w, float*& b) {
  if (s.last - s.first <= int64_t(1) << out.shift) {
    w = out.dw ? out.dw + s.group * out.ldw : nullptr;
    b = out.db ? out.db + s.group * out.ldb : nullptr;
  } else {
    w = out.partial + 2 * number * d;
    b = w + d;
  }
}

// dx of a slice's rows, and sums of dy xhat and dy over them: every thread keeps those of its columns while the rows pass.
// Sums of a block's wavefronts are joined in LDS, those of a group's slices by k_norm_join.
template <typename T, int TPR, int NV, int BLOCK>
__global__ void __launch_bounds__(BLOCK) k_norm_back(const int64_t* offsets, int64_t groups, int64_t rows, const T* dy, int64_t ldy, const T* x, int64_t ldx,
                                                     const float* weight, const float* mean, const float* rstd, int d, T* dx, int64_t ldd, Columns out) {
  constexpr int E = Vec<T>::kElems, PER = BLOCK / TPR;
  __shared__ float lds[32];
  __shared__ float join[PER > 1 ? (PER - 1) * TPR * NV * E : 1];
  const Slice s = find_slice(offsets, groups, rows, 1, out.shift, blockIdx.x);
  if (s.group < 0) return;
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float w[NV][E], sw[NV][E], sb[NV][E];
  load_columns<NV, E, TPR>(weight, 1.f, t, d, w);
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < E; ++j) sw[i][j] = sb[i][j] = 0.f;
  Vec<T> nx[NV], ny[NV];
  float nm, nr;
  const auto load = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      nx[i].load(x + row * ldx + (i * TPR + t) * E, d - (i * TPR + t) * E);
      ny[i].load(dy + row * ldy + (i * TPR + t) * E, d - (i * TPR + t) * E);
    }
    nm = mean[row];
    nr = rstd[row];
  };
  if (s.begin + sub < s.end) load(s.begin + sub);
  for (int64_t row = s.begin + sub; row < s.end; row += PER) {
    Vec<T> vx[NV], vy[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      vx[i] = nx[i];
      vy[i] = ny[i];
    }
    const float m = nm, r = nr;
    if (row + PER < s.end) load(row + PER);              // (on its way while this row is worked on)
    float a = 0.f, q = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < E; ++j) {
        // (0 behind the row's end, h too: m r alone may pass the largest number)
        const float g = vy[i].get(j), h = (i * TPR + t) * E + j < d ? (vx[i].get(j) - m) * r : 0.f;
        const float c = g * w[i][j];
        a += c;
        q = fmaf(c, h, q);
        sw[i][j] = fmaf(g, h, sw[i][j]);
        sb[i][j] += g;
      }
    row_sums<TPR, BLOCK>(a, q, lds);
    a *= -r / d;
    q *= -r / d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      vx[i].again();
      vy[i].again();
      float f[E];
#pragma unroll
      for (int j = 0; j < E; ++j) f[j] = fmaf(vy[i].get(j) * w[i][j], r, fmaf((vx[i].get(j) - m) * r, q, a));
      Vec<T> o;
      o.put(f);
      o.store(dx + row * ldd + (i * TPR + t) * E, d - (i * TPR + t) * E);
    }
  }
  float *ow, *ob;
  places(out, s, blockIdx.x, d, ow, ob);
  const auto finish = [&](float (&sum)[NV][E], float* to) {
    if constexpr (PER > 1) {
      __syncthreads();
      if (sub > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < E; ++j) join[(((sub - 1) * NV + i) * E + j) * TPR + t] = sum[i][j];
      }
      __syncthreads();
      if (sub > 0) return;
#pragma unroll 1
      for (int u = 0; u < PER - 1; ++u)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < E; ++j) sum[i][j] += join[((u * NV + i) * E + j) * TPR + t];
    }
    if (!to) return;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < E; ++j)
        if ((i * TPR + t) * E + j < d) to[(i * TPR + t) * E + j] = sum[i][j];
  };
  finish(sw, ow);
  finish(sb, ob);
}

// Rows longer than registers hold: dx row by row, and the sums by blocks of 256 columns of a slice.  16384 x 12288 fp32 993 us (2.4 TB/s
// of dy, x and dx once).
template <typename T>
__global__ void __launch_bounds__(1024) k_norm_long_dx(const int64_t* offsets, int64_t groups, int64_t rows, const T* dy, int64_t ldy, const T* x, int64_t ldx,
                                                       const float* weight, const float* mean, const float* rstd, int d, T* dx, int64_t ldd) {
  __shared__ float lds[32];
  const int64_t first = offsets ? offset_at(offsets, 0, rows) : 0, last = offsets ? offset_at(offsets, groups, rows) : rows;
  for (int64_t row = first + blockIdx.x; row < last; row += gridDim.x) {
    const T* xr = x + row * ldx;
    const T* yr = dy + row * ldy;
    T* o = dx + row * ldd;
    const float m = mean[row], r = rstd[row];
    float a = 0.f, q = 0.f;
    for (int c = threadIdx.x; c < d; c += 1024) {
      const float g = to_float(yr[c]) * (weight ? weight[c] : 1.f);
      a += g;
      q += g * ((to_float(xr[c]) - m) * r);
    }
    row_sums<1024, 1024>(a, q, lds);
    a /= d;
    q /= d;
    for (int c = threadIdx.x; c < d; c += 1024) {
      const float g = to_float(yr[c]) * (weight ? weight[c] : 1.f);
      o[c] = from_float<T>(r * (g - a - (to_float(xr[c]) - m) * r * q));
    }
  }
}
template <typename T>
__global__ void __launch_bounds__(256) k_norm_long_sums(const int64_t* offsets, int64_t groups, int64_t rows, const T* dy, int64_t ldy, const T* x, int64_t ldx,
                                                        const float* mean, const float* rstd, int d, Columns out) {
  const int across = (d + 255) / 256;
  const int64_t number = blockIdx.x / across;
  const Slice s = find_slice(offsets, groups, rows, 1, out.shift, number);
  const int c = blockIdx.x % across * 256 + threadIdx.x;
  if (s.group < 0 || c >= d) return;
  float sw = 0.f, sb = 0.f;
  for (int64_t row = s.begin; row < s.end; ++row) {
    const float g = to_float(dy[row * ldy + c]);
    sw += g * ((to_float(x[row * ldx + c]) - mean[row]) * rstd[row]);
    sb += g;
  }
  float *ow, *ob;
  places(out, s, number, d, ow, ob);
  if (ow) ow[c] = sw;
  if (ob) ob[c] = sb;
}

// Sums of the slices of every group that has several.  32 columns by 32 threads that share the slices (1024 slices of 2048 columns:
// 11 us; one thread to a column would wait for each in turn).
__global__ void __launch_bounds__(1024) k_norm_join(const int64_t* offsets, int64_t rows, int d, Columns out) {
  __shared__ double part[32][33];
  const int64_t g = blockIdx.y;
  const int64_t first = offsets ? offset_at(offsets, g, rows) : 0;
  int64_t last = offsets ? offset_at(offsets, g + 1, rows) : rows;
  if (last < first) last = first;
  const int64_t count = (last - first + (int64_t(1) << out.shift) - 1) >> out.shift;
  if (count <= 1) return;
  const int lane = threadIdx.x % 32, turn = threadIdx.x / 32, c = blockIdx.x * 32 + lane;
  const float* from = out.partial + 2 * first_number(first, g, out.shift) * d;
  for (int which = 0; which < 2; ++which) {
    float* to = which ? (out.db ? out.db + g * out.ldb : nullptr) : (out.dw ? out.dw + g * out.ldw : nullptr);
    double sum = 0;
    if (c < d) {
#pragma unroll 4
      for (int64_t j = turn; j < count; j += 32) sum += (double)from[(2 * j + which) * d + c];
    }
    __syncthreads();
    part[turn][lane] = sum;
    __syncthreads();
    if (turn == 0 && c < d && to) {
      for (int u = 1; u < 32; ++u) sum += part[u][lane];
      to[c] = (float)sum;
    }
  }
}

constexpr int64_t kDropBlocks = 8192;
constexpr int64_t kNormBlocks = 2048;      // eight to a compute unit; they go over the rows in turns

// Rows of a slice: some 1024 slices, four blocks to a compute unit, or as many as there are groups.
int slice_shift(int64_t rows) {
  int shift = 2;
  while ((rows >> shift) > 1024) ++shift;
  return shift;
}

// f(threads of a row, vectors of a thread, threads of a block) for the least that hold d columns; false if none does.
template <int E, typename F>
bool by_width(int64_t d, F f) {
#define ADACGD_WIDTH(TPR, NV, BLOCK)                                                                              \
  if (d <= TPR * NV * E) { f(std::integral_constant<int, TPR>(), std::integral_constant<int, NV>(), std::integral_constant<int, BLOCK>()); return true; }
  ADACGD_WIDTH(16, 1, 256)
  ADACGD_WIDTH(16, 2, 256)
  ADACGD_WIDTH(64, 1, 256)
  ADACGD_WIDTH(64, 2, 256)
  ADACGD_WIDTH(256, 1, 256)
  ADACGD_WIDTH(256, 2, 256)
  ADACGD_WIDTH(512, 2, 512)
  ADACGD_WIDTH(1024, 2, 1024)
#undef ADACGD_WIDTH
  return false;
}

// One block of Philox gives the draws of eight neighbouring elements (16 bits each); a thread does those eight.  They begin at
// multiples of eight of the element's number, wherever these lie in memory.  Rows that follow each other without gaps are one row.
// Bound by memory: 65536 x 2048 bf16 with a residual 149 us (5.4 TB/s), without one 96; a copy reaches 5.1.  One element a thread, and
// a generator block for each, took 500.
template <typename T>
__global__ void __launch_bounds__(256) k_dropout(const T* x, int64_t ldx, const T* residual, int64_t ldr, T* out, int64_t ldo, int64_t rows, int64_t d,
                                                 uint32_t cut, float scale, uint64_t seed, uint32_t step, const int64_t* step_dev, uint32_t layer,
                                                 uint64_t first) {
  constexpr int E = Vec<T>::kElems, V = 8 / E;
  if (step_dev) step += (uint32_t)*step_dev;
  for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
    const uint64_t e0 = first + (uint64_t)(row * d);
    const T* xr = x + row * ldx;
    const T* rr = residual + row * ldr;
    T* o = out + row * ldo;
    const int64_t groups = (int64_t)((e0 & 7) + (uint64_t)d + 7 >> 3);
    for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < groups; g += (int64_t)gridDim.x * 256) {
      const int64_t c = g * 8 - (int64_t)(e0 & 7);             // column of the first of the eight
      const uint64_t n = (e0 >> 3) + (uint64_t)g;
      const bool whole = c >= 0 && c + 8 <= d;
      Vec<T> v[V], r[V];
      if (whole) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          v[i].load(xr + c + i * E, E);
          if (residual) r[i].load(rr + c + i * E, E);
        }
      }
      uint32_t w[4];
      philox4x32_10((uint32_t)n, (uint32_t)(n >> 32), step, layer + 1, (uint32_t)seed, (uint32_t)(seed >> 32), w);
      if (whole) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float f[E];
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const int k = i * E + j;
            const uint32_t draw = k & 1 ? w[k / 2] >> 16 : w[k / 2] & 0xffff;
            f[j] = draw >= cut ? v[i].get(j) * scale : 0.f;
            if (residual) f[j] += r[i].get(j);
          }
          v[i].put(f);
          v[i].store(o + c + i * E, E);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (c + k < 0 || c + k >= d) continue;
          const uint32_t draw = k & 1 ? w[k / 2] >> 16 : w[k / 2] & 0xffff;
          float f = draw >= cut ? to_float(xr[c + k]) * scale : 0.f;
          if (residual) f += to_float(rr[c + k]);
          o[c + k] = from_float<T>(f);
        }
      }
    }
  }
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
  // (it is added to var in fp32: what that type has no number for would act as another one)
  if (!std::isfinite((float)eps) || eps < 0 || (eps > 0 && (float)eps == 0.f)) return fail(ADACGD_ERR_ARG, "eps must be finite and >= 0 in fp32");
  if (!mean != !rstd) return fail(ADACGD_ERR_ARG, "mean and rstd are given together or not at all");
  if (rows == 0) return ADACGD_OK;
  return by_dtype(x->dtype, [&](auto t) {
    using T = decltype(t);
    const bool held = by_width<Vec<T>::kElems>(d, [&](auto tpr, auto nv, auto block) {
      const int64_t blocks = (rows + block / tpr - 1) / (block / tpr);
      k_norm<T, tpr, nv, block><<<blocks < kNormBlocks ? blocks : kNormBlocks, block.value, 0, (hipStream_t)stream>>>(
          (const T*)x->data, x->stride, weight, bias, rows, (int)d, (float)eps, (T*)y->data, y->stride, mean, rstd);
    });
    if (!held)
      k_norm_long<T><<<rows < kNormBlocks ? rows : kNormBlocks, 1024, 0, (hipStream_t)stream>>>((const T*)x->data, x->stride, weight, bias, rows, (int)d, (float)eps, (T*)y->data,
                                                                                               y->stride, mean, rstd);
    return launched("adacgd_layer_norm");
  });
}

int adacgd_layer_norm_backward_workspace_bytes(int64_t rows, int64_t groups, int64_t d, int64_t* bytes) {
  if (!bytes) return fail(ADACGD_ERR_ARG, "bytes is null");
  ADACGD_TRY(check_count("rows", rows, 0, kMaxCount));
  ADACGD_TRY(check_count("groups", groups, 1, 65535));
  ADACGD_TRY(check_count("d", d, 1, kMaxColumns));
  const int shift = slice_shift(rows);
  // (a group of that many rows at most is one slice)
  *bytes = rows <= int64_t(1) << shift ? 0 : (slice_numbers(rows, groups, shift) * 2 * d * 4 + 255) / 256 * 256;
  return ADACGD_OK;
}

int adacgd_layer_norm_backward(int64_t rows, int64_t groups, int64_t d, const int64_t* offsets, const adacgd_tensor* dy,
                               const adacgd_tensor* x, const float* weight, const float* mean, const float* rstd,
                               const adacgd_tensor* dx, const adacgd_tensor* dweight, const adacgd_tensor* dbias,
                               void* workspace, int64_t workspace_bytes, void* stream) {
  int64_t need = 0;
  ADACGD_TRY(adacgd_layer_norm_backward_workspace_bytes(rows, groups, d, &need));
  if (!offsets && groups != 1) return fail(ADACGD_ERR_ARG, "offsets is null, but there are %lld groups", (long long)groups);
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
  if (rows == 0 && !dweight && !dbias) return ADACGD_OK;
  const int shift = slice_shift(rows);
  const Columns out{dweight ? (float*)dweight->data : nullptr, dbias ? (float*)dbias->data : nullptr, dweight ? dweight->stride : 0, dbias ? dbias->stride : 0,
                    (float*)workspace, shift};
  const int64_t numbers = slice_numbers(rows, groups, shift);
  return by_dtype(x->dtype, [&](auto t) -> int {
    using T = decltype(t);
    const bool held = by_width<Vec<T>::kElems>(d, [&](auto tpr, auto nv, auto block) {
      k_norm_back<T, tpr, nv, block><<<numbers, block.value, 0, (hipStream_t)stream>>>(offsets, groups, rows, (const T*)dy->data, dy->stride, (const T*)x->data, x->stride, weight,
                                                                               mean, rstd, (int)d, (T*)dx->data, dx->stride, out);
    });
    if (!held) {
      if (rows > 0)
        k_norm_long_dx<T><<<rows < kNormBlocks ? rows : kNormBlocks, 1024, 0, (hipStream_t)stream>>>(offsets, groups, rows, (const T*)dy->data, dy->stride, (const T*)x->data,
                                                                                                   x->stride, weight, mean, rstd, (int)d, (T*)dx->data, dx->stride);
      const int64_t blocks = (d + 255) / 256 * numbers;
      if (blocks > kMaxCount / 256) return fail(ADACGD_ERR_ARG, "more columns and groups than one launch takes");
      if (dweight || dbias)
        k_norm_long_sums<T><<<blocks, 256, 0, (hipStream_t)stream>>>(offsets, groups, rows, (const T*)dy->data, dy->stride, (const T*)x->data, x->stride,
                                                                                          mean, rstd, (int)d, out);
    }
    if (rows > int64_t(1) << shift && (dweight || dbias)) k_norm_join<<<dim3((d + 31) / 32, groups), 1024, 0, (hipStream_t)stream>>>(offsets, rows, (int)d, out);
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
  if (first + (uint64_t)(rows * d - 1) < first) return fail(ADACGD_ERR_ARG, "first and the elements pass 2^64");
  const uint32_t cut = (uint32_t)std::floor(p * 65536 + 0.5);
  const float scale = cut == 65536 ? 0.f : (float)(65536.0 / (65536 - cut));
  if (rows > 1 && x->stride == d && out->stride == d && (!residual || residual->stride == d)) { d *= rows; rows = 1; }
  const int64_t across = (d + 14) / 8 / 256 + 1;
  const dim3 grid(across < kDropBlocks ? across : kDropBlocks, rows < 32768 ? rows : 32768);
  return by_dtype(x->dtype, [&](auto t) {
    using T = decltype(t);
    k_dropout<T><<<grid, 256, 0, (hipStream_t)stream>>>((const T*)x->data, x->stride, residual ? (const T*)residual->data : nullptr, residual ? residual->stride : 0,
                                                        (T*)out->data, out->stride, rows, d, cut, scale, seed, step, step_dev, layer, first);
    return launched("adacgd_dropout");
  });
}

}  // extern "C"
