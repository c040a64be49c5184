// Preference loss of paired sequences' log ratios, from logits, and its gradient.
#include <cmath>

#include "layers.h"

namespace adacgd {
namespace {

constexpr int64_t kMaxPairs = 1 << 22;      // (one launch takes 2^32 threads)
constexpr float kLog2e = 1.4426950408889634f, kLog2eLow = 1.925963033500929e-8f;      // log2(e) and what the first leaves of it

struct Lse { float top, sum; };       // sum of exp(x - top)
__device__ __forceinline__ Lse join(Lse a, Lse b) {
  const float top = fmaxf(a.top, b.top);
  // (a part without elements, or of nothing but -inf, has sum 0; a row's other infinities give the NaN that the definition gives)
  const float fa = a.sum == 0.f ? 0.f : a.sum * expf(a.top - top), fb = b.sum == 0.f ? 0.f : b.sum * expf(b.top - top);
  return Lse{top, fa + fb};
}
// exp(x - y) by the instruction for powers of two.  x - y is formed before the factor of the base: near the largest elements, which
// make up the sum, it has no error.  The factor's own rounding (1.3e-8 of it) would make every term too large: sums were off by
// 5e-8 on average, and a pair's margin by that times the difference of its sequences' lengths.
__device__ __forceinline__ float exp_diff(float x, float y) {
  const float d = x - y;
  return __builtin_amdgcn_exp2f(fmaf(d, kLog2e, d * kLog2eLow));
}

// A row is split into parts where there are few rows, so that 1024 blocks are at work (4096 were no faster); each part is whole vectors
// of a block.
struct Parts {
  int64_t count, length;
};
constexpr int kUnroll = 4;      // vectors of a thread on their way
constexpr int64_t kTokenBlocks = 1024;
// Where every part of a row reads all of it for its sum (k_token_grad): 61 rows of 128000 fp32 30 us (44 by 1024 blocks), 250 58 (113).
constexpr int64_t kSumBlocks = 256;
inline Parts parts_of(int64_t tokens, int64_t v, int64_t blocks = kTokenBlocks) {
  const int64_t unit = 2048;
  int64_t count = tokens > 0 ? blocks / tokens : 1;
  const int64_t most = (v + unit - 1) / unit;
  count = count < 1 ? 1 : count > most ? most : count;
  const int64_t length = ((v + count - 1) / count + unit - 1) / unit * unit;
  return Parts{(v + length - 1) / length, length};
}
inline bool narrow(int64_t v) { return v <= 8192; }      // a wavefront to a row (4096 logits: 54 us, 104 by 256 threads), else 256 threads

// Largest element and sum of exponentials of (a part of) every row that counts, in one pass: a thread's sum is scaled down
// when one of its vectors has a larger element.  The target's logit is put aside by the part that has it.  Bound by memory where
// a row is long: 8192 x 32000 bf16 110 to 116 us (4.5 to 4.8 TB/s; in two passes over a row 479), 32768 x 4096 by a wavefront each 54 (by 256
// threads 104); 10^5 rows of 250 wait for the chain of target, row and sum: 72 us, 0.7 TB/s.
template <typename T, int TPR>
__global__ void __launch_bounds__(256) k_token(int64_t tokens, int64_t sequences, int64_t v, const T* logits, int64_t ld, const int64_t* targets, const int64_t* offsets,
                                               Parts parts, Lse* out, float* at_target) {
  constexpr int E = Vec<T>::kElems, PER = 256 / TPR;
  __shared__ Lse part[4];
  const int t0 = threadIdx.x % TPR;
  const int64_t first = offset_at(offsets, 0, tokens), last = offset_at(offsets, sequences, tokens);
  for (int64_t u = (int64_t)blockIdx.x * PER + threadIdx.x / TPR; u < tokens * parts.count; u += (int64_t)gridDim.x * PER) {
    const int64_t t = u / parts.count, begin = (u - t * parts.count) * parts.length;
    if (t < first || t >= last) continue;
    const int64_t target = targets[t];
    if (target < 0 || target >= v) continue;
    const int64_t end = begin + parts.length < v ? begin + parts.length : v;
    const T* row = logits + t * ld;
    if (t0 == 0 && target >= begin && target < end) at_target[t] = to_float(row[target]);
    Lse l{-INFINITY, 0.f};
    const auto take = [&](const Vec<T>& q) {
      float top = q.get(0);
#pragma unroll
      for (int j = 1; j < E; ++j) top = fmaxf(top, q.get(j));
      if (top > l.top) {
        if (l.sum != 0.f) l.sum *= exp_diff(l.top, top);
        l.top = top;
      }
      const float base = l.top == -INFINITY ? 0.f : l.top;
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < E; ++j) s += exp_diff(q.get(j), base);
      l.sum += s;
    };
    int64_t c = begin + t0 * E;
    for (; c + (kUnroll - 1) * TPR * E + E <= end; c += kUnroll * TPR * E) {
      Vec<T> q[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) q[k].load(row + c + k * TPR * E, E);
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) take(q[k]);
    }
    for (; c < end; c += TPR * E) {
      Vec<T> q;
      q.load(row + c, end - c, -INFINITY);
      take(q);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) l = join(l, Lse{__shfl_xor(l.top, o, 64), __shfl_xor(l.sum, o, 64)});
    if constexpr (TPR > 64) {
      if (lane_id() == 0) part[threadIdx.x / 64] = l;
      __syncthreads();
      if (t0 == 0)
        for (int w = 1; w < 4; ++w) l = join(l, part[w]);
      __syncthreads();
    }
    if (t0 == 0) out[u] = l;
  }
}

// Log-probabilities of a pair's tokens, the sums of their differences from the reference, and the loss.  Bound by the longest pair, which is
// one block's: with k_token, 32768 tokens of 250 logits in one pair take 78 us, in sixteen 27.
constexpr int kPairThreads = 512;
__global__ void __launch_bounds__(kPairThreads) k_pair(int64_t tokens, int64_t v, const int64_t* targets, const int64_t* offsets, int64_t parts, const Lse* in, const float* at_target,
                                                       const float* ref, double beta, double smoothing, float* loss, float* margin, float* logp, float* lse) {
  __shared__ double sums[kPairThreads / 64];
  const int64_t p = blockIdx.x;
  const int64_t first = offset_at(offsets, 2 * p, tokens), middle = offset_at(offsets, 2 * p + 1, tokens), last = offset_at(offsets, 2 * p + 2, tokens);
  double s = 0;
#pragma unroll 2
  for (int64_t t = first + threadIdx.x; t < last; t += kPairThreads) {
    const int64_t target = targets[t];
    double lp = 0, l = 0;
    if (target >= 0 && target < v) {
      Lse a = in[t * parts];
      for (int64_t k = 1; k < parts; ++k) a = join(a, in[t * parts + k]);
      const double ls = log((double)a.sum);
      l = a.top + ls;
      lp = ((double)at_target[t] - (double)a.top) - ls;
      const double ratio = lp - (ref ? (double)ref[t] : 0.0);
      s += t < middle ? ratio : -ratio;
    }
    logp[t] = (float)lp;
    lse[t] = (float)l;
  }
  s = wave_sum(s);
  if (lane_id() == 0) sums[threadIdx.x / 64] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double m = sums[0];
    for (int w = 1; w < kPairThreads / 64; ++w) m += sums[w];
    const double z = beta * m, soft = log1p(exp(-fabs(z)));
    margin[p] = (float)m;
    // (a weight of zero takes its term away, an infinite one too)
    loss[p] = (float)((smoothing < 1 ? (1 - smoothing) * (soft + fmax(-z, 0.0)) : 0.0) + (smoothing > 0 ? smoothing * (soft + fmax(z, 0.0)) : 0.0));
  }
}

// dlogits of (a part of) every row: f (onehot - p), f from the margin of the row's pair, p = exp(x - lse).  lse was rounded to fp32, by
// up to 2^-24 of its own size, which is a relative error of every p of the row (and all of p where the elements are the type's
// lowest: lse has lost the logarithm of their number).  While that is at most 1/64 of what storing the result loses, |lse| <= 1024 in
// bf16 and 128 in fp16, it stays.  Otherwise, in fp32 nearly always, the row's sum is formed anew around lse, where x - lse has no
// such error, and divided by; the row is read twice then.  Bound by memory: 8192 x 32000 bf16 201 us (5.2 TB/s), 239 with the sum, fp32 478 (404
// without it).
template <typename T>
constexpr float kExactLse = __is_same(T, __bf16) ? 1024.f : sizeof(T) == 2 ? 128.f : 0.015625f;
template <typename T, int TPR>
__global__ void __launch_bounds__(256) k_token_grad(int64_t tokens, int64_t sequences, int64_t v, const float* dloss, const T* logits, int64_t ld, const int64_t* targets,
                                                    const int64_t* offsets, const float* margin, const float* lse, double beta, double smoothing, Parts parts, bool in_place, T* out, int64_t ldo) {
  constexpr int E = Vec<T>::kElems, PER = 256 / TPR;
  __shared__ float part[4];
  const int t0 = threadIdx.x % TPR;
  const int64_t first = offset_at(offsets, 0, tokens), last = offset_at(offsets, sequences, tokens);
  for (int64_t u = (int64_t)blockIdx.x * PER + threadIdx.x / TPR; u < tokens * parts.count; u += (int64_t)gridDim.x * PER) {
    const int64_t t = u / parts.count, begin = (u - t * parts.count) * parts.length;
    if (t < first || t >= last) continue;
    int64_t end = begin + parts.length < v ? begin + parts.length : v;
    const T* row = logits + t * ld;
    T* o = out + t * ldo;
    const int64_t target = targets[t];
    if (target < 0 || target >= v) {
      const Vec<T> zero{word4{0, 0, 0, 0}};
      for (int64_t c = begin + t0 * E; c < end; c += TPR * E) zero.store(o + c, end - c);
      continue;
    }
    const int64_t low = group_of(offsets, sequences, tokens, t);
    // (of the margin as the caller has it, in fp32: a relative error of |z| 2^-24 at most in either term of the slope)
    const double z = beta * (double)margin[low / 2];
    const double slope = (smoothing / (1 + exp(-z)) - (1 - smoothing) / (1 + exp(z))) * beta * (double)dloss[low / 2];
    const float f = (float)(low % 2 ? -slope : slope), l = lse[t];
    float fs = f;                                            // f / (sum of exp(x - l))
    if (!(fabsf(l) <= kExactLse<T>)) {                       // (all threads of a row's parts alike)
      if (in_place) {                                          // the other parts must not be written before they are read here
        if (begin > 0) continue;
        end = v;
      }
      float sum = 0.f;
      const auto add = [&](const Vec<T>& q) {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < E; ++j) s += exp_diff(q.get(j), l);
        sum += s;
      };
      int64_t c = t0 * E;
      for (; c + (kUnroll - 1) * TPR * E + E <= v; c += kUnroll * TPR * E) {
        Vec<T> q[kUnroll];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) q[k].load(row + c + k * TPR * E, E);
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) add(q[k]);
      }
      for (; c < v; c += TPR * E) {
        Vec<T> q;
        q.load(row + c, v - c, -INFINITY);
        add(q);
      }
      sum = wave_sumf(sum);
      if constexpr (TPR > 64) {
        if (lane_id() == 0) part[threadIdx.x / 64] = sum;
        __syncthreads();                                      // (the row has been read, and may be written)
        sum = part[0];
        for (int w = 1; w < 4; ++w) sum += part[w];
        __syncthreads();
      }
      fs = f / sum;
    }
    const auto take = [&](Vec<T>& q, int64_t c) {
      float g[E];
#pragma unroll
      for (int j = 0; j < E; ++j) g[j] = fmaf(exp_diff(q.get(j), l), -fs, c + j == target ? f : 0.f);
      q.put(g);
    };
    int64_t c = begin + t0 * E;
    for (; c + (kUnroll - 1) * TPR * E + E <= end; c += kUnroll * TPR * E) {
      Vec<T> q[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) q[k].load(row + c + k * TPR * E, E);
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        take(q[k], c + k * TPR * E);
        q[k].store(o + c + k * TPR * E, E);
      }
    }
    for (; c < end; c += TPR * E) {
      Vec<T> q;
      q.load(row + c, end - c);
      take(q, c);
      q.store(o + c, end - c);
    }
  }
}
inline int64_t token_blocks(int64_t units) { return units < (int64_t(1) << 20) ? units : int64_t(1) << 20; }

// Workspace: sums of the parts of rows, then the targets' logits.
inline int64_t sums_bytes(int64_t tokens, int64_t v) { return (tokens * parts_of(tokens, v).count * (int64_t)sizeof(Lse) + 255) / 256 * 256; }

int check_common(int64_t tokens, int64_t pairs, int64_t v, const adacgd_tensor* logits, const int64_t* targets, const int64_t* offsets, double beta, double smoothing) {
  ADACGD_TRY(check_count("tokens", tokens, 0, kMaxCount));
  ADACGD_TRY(check_count("pairs", pairs, 0, kMaxPairs));
  ADACGD_TRY(check_count("v", v, 1, kMaxColumns));
  ADACGD_TRY(check_tensor(logits, "logits", tokens, v, false, false));
  if (tokens > 0 && !targets) return fail(ADACGD_ERR_ARG, "targets is null");
  if (!offsets) return fail(ADACGD_ERR_ARG, "offsets is null");
  if (!std::isfinite(beta)) return fail(ADACGD_ERR_ARG, "beta must be finite");
  if (!(smoothing >= 0 && smoothing <= 1)) return fail(ADACGD_ERR_ARG, "smoothing must be in [0, 1]");
  return ADACGD_OK;
}

}  // namespace
}  // namespace adacgd

using namespace adacgd;

extern "C" {

int adacgd_preference_loss_workspace_bytes(int64_t tokens, int64_t pairs, int64_t v, int64_t* bytes) {
  if (!bytes) return fail(ADACGD_ERR_ARG, "bytes is null");
  ADACGD_TRY(check_count("tokens", tokens, 0, kMaxCount));
  ADACGD_TRY(check_count("pairs", pairs, 0, kMaxPairs));
  ADACGD_TRY(check_count("v", v, 1, kMaxColumns));
  *bytes = sums_bytes(tokens, v) + (tokens * (int64_t)sizeof(float) + 255) / 256 * 256;
  return ADACGD_OK;
}

int adacgd_preference_loss(int64_t tokens, int64_t pairs, int64_t v, const adacgd_tensor* logits, const int64_t* targets,
                           const int64_t* offsets, const float* ref, double beta, double smoothing, float* loss,
                           float* margin, float* logp, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  ADACGD_TRY(check_common(tokens, pairs, v, logits, targets, offsets, beta, smoothing));
  if (pairs > 0 && (!loss || !margin)) return fail(ADACGD_ERR_ARG, "loss or margin is null");
  if (tokens > 0 && (!logp || !lse)) return fail(ADACGD_ERR_ARG, "logp or lse is null");
  int64_t need = 0;
  ADACGD_TRY(adacgd_preference_loss_workspace_bytes(tokens, pairs, v, &need));
  ADACGD_TRY(check_workspace(workspace, workspace_bytes, need));
  if (pairs == 0) return ADACGD_OK;
  return by_dtype(logits->dtype, [&](auto t) -> int {
    using T = decltype(t);
    const Parts parts = parts_of(tokens, v);
    Lse* sums = (Lse*)workspace;
    float* at_target = (float*)((char*)workspace + sums_bytes(tokens, v));
    const int64_t units = tokens * parts.count;
    const hipStream_t on = (hipStream_t)stream;
    if (tokens > 0) {
      if (narrow(v))
        k_token<T, 64><<<token_blocks((units + 3) / 4), 256, 0, on>>>(tokens, 2 * pairs, v, (const T*)logits->data, logits->stride, targets, offsets, parts, sums, at_target);
      else
        k_token<T, 256><<<token_blocks(units), 256, 0, on>>>(tokens, 2 * pairs, v, (const T*)logits->data, logits->stride, targets, offsets, parts, sums, at_target);
      ADACGD_TRY(launched("adacgd_preference_loss"));
    }
    k_pair<<<pairs, kPairThreads, 0, on>>>(tokens, v, targets, offsets, parts.count, sums, at_target, ref, beta, smoothing, loss, margin, logp, lse);
    return launched("adacgd_preference_loss");
  });
}

int adacgd_preference_loss_backward(int64_t tokens, int64_t pairs, int64_t v, const float* dloss, const adacgd_tensor* logits,
                                    const int64_t* targets, const int64_t* offsets, const float* margin, const float* lse,
                                    double beta, double smoothing, const adacgd_tensor* dlogits, void* stream) {
  ADACGD_TRY(check_common(tokens, pairs, v, logits, targets, offsets, beta, smoothing));
  ADACGD_TRY(check_tensor(dlogits, "dlogits", tokens, v, false, false));
  if (logits->dtype != dlogits->dtype) return fail(ADACGD_ERR_ARG, "logits and dlogits differ in type");
  if (tokens == 0 || pairs == 0) return ADACGD_OK;
  if (!dloss || !margin || !lse) return fail(ADACGD_ERR_ARG, "dloss, margin or lse is null");
  return by_dtype(logits->dtype, [&](auto t) {
    using T = decltype(t);
    const Parts parts = parts_of(tokens, v, sizeof(T) == 4 ? kSumBlocks : kTokenBlocks);
    const int64_t units = tokens * parts.count;
    const auto go = [&](auto kernel, int64_t blocks) {
      kernel<<<token_blocks(blocks), 256, 0, (hipStream_t)stream>>>(tokens, 2 * pairs, v, dloss, (const T*)logits->data, logits->stride, targets, offsets, margin, lse, beta, smoothing,
                                                                    parts, dlogits->data == logits->data, (T*)dlogits->data, dlogits->stride);
    };
    if (narrow(v)) go(k_token_grad<T, 64>, (units + 3) / 4);
    else go(k_token_grad<T, 256>, units);
    return launched("adacgd_preference_loss_backward");
  });
}

}  // extern "C"
