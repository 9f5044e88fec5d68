// bakron_token_logprobs and bakron_token_logprobs_backward.
//
//   lse = m + log(sum exp(l - m)),  logp = l[target] - lse,  H = lse - sum p l
//   dl_j = g ([j = target] - p_j) - u p_j (log p_j + H)
#include <limits.h>

#include "rowops.cuh"

namespace bakron {
namespace {

constexpr int TOP_MAX = 32;
constexpr float LSE_EXACT = 1024.f;   // up to here lse's rounding is below 2^-14

struct LogprobParams {
  const void* logits;
  int64_t ld;
  const int64_t* targets;
  int rows, v, top;
  float *logp, *entropy, *lse, *top_logp;
  int* top_ids;
};

struct MaxOp {
  __device__ __forceinline__ float operator()(float a, float b) const { return max_nan(a, b); }
  static constexpr float none = -INFINITY;
};

// The larger value first, the lower index first among equal ones.
__device__ __forceinline__ bool before(float a, int i, float b, int j) {
  return a > b || (a == b && i < j);
}

template <typename T>
__global__ void __launch_bounds__(256) k_logprob(const LogprobParams P) {
  __shared__ float slots[4][32];
  __shared__ float bv[8];
  __shared__ int bi[8];
  const int64_t row = blockIdx.x;
  const T* l = (const T*)P.logits + row * P.ld;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float m = -INFINITY;
  for (int e = threadIdx.x; e < P.v; e += 256) m = max_nan(m, to_f32(l[e]));
  m = cta_all(m, MaxOp(), slots[0]);
  const bool none = m == -INFINITY;
  float s = 0.f, u = 0.f;
  for (int e = threadIdx.x; e < P.v; e += 256) {
    const float t = to_f32(l[e]) - m, p = expf(t);
    s += p;
    u += p == 0.f ? 0.f : p * t;
  }
  s = cta_all(s, AddOp(), slots[1]);
  u = cta_all(u, AddOp(), slots[2]);
  const float lse = none ? -INFINITY : m + logf(s);
  if (threadIdx.x == 0) {
    const int64_t at = P.targets ? P.targets[row] : -1;
    P.lse[row] = lse;
    P.entropy[row] = none ? 0.f : logf(s) - u / s;
    if (P.logp)
      P.logp[row] = at < 0 || at >= P.v ? 0.f : none ? -INFINITY : (to_f32(l[at]) - m) - logf(s);
  }
  float pv = INFINITY;
  int pi = -1;
  for (int k = 0; k < P.top; ++k) {   // the best one after (pv, pi)
    float v = -INFINITY;
    int i = INT_MAX;
    for (int e = threadIdx.x; e < P.v; e += 256) {
      const float x = to_f32(l[e]);
      if (before(pv, pi, x, e) && before(x, e, v, i)) {
        v = x;
        i = e;
      }
    }
    for (int o = 16; o; o >>= 1) {
      const float ov = __shfl_xor_sync(0xffffffffu, v, o);
      const int oi = __shfl_xor_sync(0xffffffffu, i, o);
      if (before(ov, oi, v, i)) {
        v = ov;
        i = oi;
      }
    }
    if (lane == 0) {
      bv[warp] = v;
      bi[warp] = i;
    }
    __syncthreads();
    v = bv[0];
    i = bi[0];
    for (int w = 1; w < 8; ++w)
      if (before(bv[w], bi[w], v, i)) {
        v = bv[w];
        i = bi[w];
      }
    __syncthreads();
    if (threadIdx.x == 0) {
      P.top_logp[row * P.top + k] = none ? -INFINITY : (v - m) - logf(s);
      P.top_ids[row * P.top + k] = i == INT_MAX ? -1 : i;
    }
    pv = v;
    pi = i;
  }
}

struct LogprobBackParams {
  const void* logits;
  int64_t ld, ldd;
  const int64_t* targets;
  const float *lse, *entropy, *dlogp, *dentropy;
  void* d;
  int rows, v;
};

template <typename T>
__global__ void __launch_bounds__(256) k_logprob_back(const LogprobBackParams P) {
  __shared__ float slots[2][32];
  const int64_t row = blockIdx.x;
  const T* l = (const T*)P.logits + row * P.ld;
  T* d = (T*)P.d + row * P.ldd;
  const int64_t at = P.targets ? P.targets[row] : -1;
  const float lse = P.lse[row];
  const float g = P.dlogp && at >= 0 && at < P.v ? P.dlogp[row] : 0.f;
  const float u = P.dentropy ? P.dentropy[row] : 0.f, H = P.dentropy ? P.entropy[row] : 0.f;
  const bool none = lse == -INFINITY;
  // log p = (l - m) - log s.  lse = m + log s in one number is enough unless it is so
  // large that its rounding is felt: such a row's m and s are formed again.
  float m = lse, ls = 0.f;
  if (fabsf(lse) > LSE_EXACT && !none) {
    m = -INFINITY;
    for (int e = threadIdx.x; e < P.v; e += 256) m = max_nan(m, to_f32(l[e]));
    m = cta_all(m, MaxOp(), slots[0]);
    for (int e = threadIdx.x; e < P.v; e += 256) ls += expf(to_f32(l[e]) - m);
    ls = logf(cta_all(ls, AddOp(), slots[1]));
  }
  for (int e = threadIdx.x; e < P.v; e += 256) {
    const float t = (to_f32(l[e]) - m) - ls, p = expf(t);
    float v = -g * p;
    if (p != 0.f) v -= u * p * (t + H);
    if (e == at) v += g;
    d[e] = from_f32<T>(none ? 0.f : v);
  }
}

}  // namespace
}  // namespace bakron

using namespace bakron;

extern "C" int bakron_token_logprobs(const void* logits, int dtype, int rows, int v, int64_t ldl,
                                     const int64_t* targets, int top, float* logp, float* entropy,
                                     float* lse, float* top_logp, int* top_ids, void* stream) {
  if ((dtype != BAKRON_F32 && dtype != BAKRON_BF16) || rows < 0 || v < 1 || top < 0 || top > TOP_MAX ||
      top > v || (targets != nullptr) != (logp != nullptr))
    return BAKRON_ERR_INVALID_ARG;
  if (rows == 0) return BAKRON_OK;
  if (!logits || ldl < v || !entropy || !lse || (top > 0 && (!top_logp || !top_ids)))
    return BAKRON_ERR_INVALID_ARG;
  LogprobParams P{logits, ldl, targets, rows, v, top, logp, entropy, lse, top_logp, top_ids};
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == BAKRON_F32)
    k_logprob<float><<<rows, 256, 0, s>>>(P);
  else
    k_logprob<__nv_bfloat16><<<rows, 256, 0, s>>>(P);
  BK_CUDA_OK(cudaGetLastError());
  return BAKRON_OK;
}

extern "C" int bakron_token_logprobs_backward(const void* logits, int dtype, int rows, int v,
                                              int64_t ldl, const int64_t* targets, const float* lse,
                                              const float* dlogp, const float* entropy,
                                              const float* dentropy, void* dlogits, int64_t ldd,
                                              void* stream) {
  if ((dtype != BAKRON_F32 && dtype != BAKRON_BF16) || rows < 0 || v < 1) return BAKRON_ERR_INVALID_ARG;
  if (rows == 0) return BAKRON_OK;
  if (!logits || !lse || !dlogits || ldl < v || ldd < v || (!dlogp && !dentropy) ||
      (dlogp && !targets) || (dentropy && !entropy))
    return BAKRON_ERR_INVALID_ARG;
  LogprobBackParams P{logits, ldl, ldd, targets, lse, entropy, dlogp, dentropy, dlogits, rows, v};
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == BAKRON_F32)
    k_logprob_back<float><<<rows, 256, 0, s>>>(P);
  else
    k_logprob_back<__nv_bfloat16><<<rows, 256, 0, s>>>(P);
  BK_CUDA_OK(cudaGetLastError());
  return BAKRON_OK;
}
