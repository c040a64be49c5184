// Preference loss of paired sequences' log ratios, from logits, and its gradient.
#include <cmath>

#include "layers.h"

namespace adacgd {
namespace {

struct Lse { float top, sum; };       // sum of exp(x - top)
__device__ __forceinline__ Lse join(Lse a, Lse b) {
  const float top = fmaxf(a.top, b.top);
  // (a part without elements has top = -inf and sum 0; infinities of the row give the NaN that the definition gives)
  const float fa = a.sum == 0.f ? 0.f : a.sum * expf(a.top - top), fb = b.sum == 0.f ? 0.f : b.sum * expf(b.top - top);
  return Lse{top, fa + fb};
}

// Largest element and sum of exponentials of every token's row that counts.
template <typename T>
__global__ void __launch_bounds__(256) k_token(int64_t tokens, int64_t sequences, int64_t v, const T* logits, int64_t ld, const int64_t* targets, const int64_t* offsets, Lse* parts) {
  __shared__ Lse part[4];
  const int64_t t = blockIdx.x;
  if (t < offset_at(offsets, 0, tokens) || t >= offset_at(offsets, sequences, tokens)) return;
  const int64_t target = targets[t];
  if (target < 0 || target >= v) return;
  logits += t * ld;
  float top = -INFINITY;
  for (int64_t c = threadIdx.x; c < v; c += 256) top = fmaxf(top, to_float(logits[c]));
  float sum = 0.f;
  const float base = top == -INFINITY ? 0.f : top;          // (a part of nothing but -inf sums to 0)
  for (int64_t c = threadIdx.x; c < v; c += 256) sum += expf(to_float(logits[c]) - base);
  Lse l{top, sum};
  for (int o = 32; o > 0; o >>= 1) l = join(l, Lse{__shfl_xor(l.top, o, 64), __shfl_xor(l.sum, o, 64)});
  if (lane_id() == 0) part[threadIdx.x / 64] = l;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 4; ++w) l = join(l, part[w]);
    parts[t] = l;
  }
}

// Log-probabilities of a pair's tokens, the sum of their differences from the reference, and the loss.
template <typename T>
__global__ void __launch_bounds__(64) k_pair(int64_t tokens, int64_t v, const T* logits, int64_t ld, const int64_t* targets, const int64_t* offsets, const Lse* parts, const float* ref, double beta, double smoothing, float* loss, float* margin, float* logp, float* lse) {
  const int64_t p = blockIdx.x;
  double m = 0;
  for (int q = 0; q < 2; ++q) {
    const int64_t first = offset_at(offsets, 2 * p + q, tokens), last = offset_at(offsets, 2 * p + q + 1, tokens);
    double s = 0;
    for (int64_t t = first + threadIdx.x; t < last; t += 64) {
      const int64_t target = targets[t];
      double lp = 0, l = 0;
      if (target >= 0 && target < v) {
        const double ls = log((double)parts[t].sum);
        l = parts[t].top + ls;
        lp = ((double)to_float(logits[t * ld + target]) - (double)parts[t].top) - ls;
        s += lp - (ref ? (double)ref[t] : 0.0);
      }
      logp[t] = (float)lp;
      lse[t] = (float)l;
    }
    s = wave_sum(s);
    m = q ? m - s : s;
  }
  if (threadIdx.x == 0) {
    const double z = beta * m, soft = log1p(exp(-fabs(z)));
    margin[p] = (float)m;
    // (a weight of zero takes its term away, an infinite one too)
    loss[p] = (float)((smoothing < 1 ? (1 - smoothing) * (soft + fmax(-z, 0.0)) : 0.0) + (smoothing > 0 ? smoothing * (soft + fmax(z, 0.0)) : 0.0));
  }
}

template <typename T>
__global__ void __launch_bounds__(256) k_token_grad(int64_t tokens, int64_t sequences, int64_t v, const float* dloss, const T* logits, int64_t ld, const int64_t* targets, const int64_t* offsets, const float* margin, const float* lse, double beta, double smoothing, T* out, int64_t ldo) {
  const int64_t t = blockIdx.x;
  if (t < offset_at(offsets, 0, tokens) || t >= offset_at(offsets, sequences, tokens)) return;
  logits += t * ld;
  out += t * ldo;
  const int64_t target = targets[t];
  if (target < 0 || target >= v) {
    for (int64_t c = threadIdx.x; c < v; c += 256) out[c] = from_float<T>(0.f);
    return;
  }
  int64_t low = 0, count = sequences;                 // the last sequence that begins at or before t
  while (count > 1) { const int64_t h = count / 2; if (offset_at(offsets, low + h, tokens) <= t) { low += h; count -= h; } else count = h; }
  const double z = beta * (double)margin[low / 2];
  const double slope = (smoothing / (1 + exp(-z)) - (1 - smoothing) / (1 + exp(z))) * beta * (double)dloss[low / 2];
  const float f = (float)(low % 2 ? -slope : slope);
  const float l = lse[t];
  for (int64_t c = threadIdx.x; c < v; c += 256) {
    const float e = expf(to_float(logits[c]) - l);
    out[c] = from_float<T>(f * ((c == target ? 1.f : 0.f) - e));
  }
}

int check_common(int64_t tokens, int64_t pairs, int64_t v, const adacgd_tensor* logits, const int64_t* targets, const int64_t* offsets, double beta, double smoothing) {
  ADACGD_TRY(check_count("tokens", tokens, 0, kMaxCount));
  ADACGD_TRY(check_count("pairs", pairs, 0, kMaxCount / 2));
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
  ADACGD_TRY(check_count("pairs", pairs, 0, kMaxCount / 2));
  ADACGD_TRY(check_count("v", v, 1, kMaxColumns));
  *bytes = (tokens * (int64_t)sizeof(Lse) + 255) / 256 * 256;
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
    if (tokens > 0) {
      k_token<T><<<tokens, 256, 0, (hipStream_t)stream>>>(tokens, 2 * pairs, v, (const T*)logits->data, logits->stride, targets, offsets, (Lse*)workspace);
      ADACGD_TRY(launched("adacgd_preference_loss"));
    }
    k_pair<T><<<pairs, 64, 0, (hipStream_t)stream>>>(tokens, v, (const T*)logits->data, logits->stride, targets, offsets, (const Lse*)workspace, ref, beta, smoothing, loss, margin, logp, lse);
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
    k_token_grad<T><<<tokens, 256, 0, (hipStream_t)stream>>>(tokens, 2 * pairs, v, dloss, (const T*)logits->data, logits->stride, targets, offsets, margin, lse, beta, smoothing, (T*)dlogits->data, dlogits->stride);
    return launched("adacgd_preference_loss_backward");
  });
}

}  // extern "C"
