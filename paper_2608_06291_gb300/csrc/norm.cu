// bakron_rmsnorm and bakron_rmsnorm_backward.
//
//   h = x + r,  rho = 1 / sqrt(mean(h^2) + eps),  y = w h rho
//   dx = rho (w dy - h rho^2 mean(w dy h)) + dsum,  dw = sum over rows of dy h rho
//
// The sum h is formed and kept in fp32; it is rounded once where it is stored, and y
// comes from the unrounded one.
#include <float.h>

#include <algorithm>

#include "rowops.cuh"

namespace bakron {
namespace {

constexpr int NORM_MAX_D = 1 << 16;
constexpr float E4M3_MAX = 448.f;

struct NormParams {
  const void *x, *res, *w;
  int64_t ldx, ldr, ldh, ldy;
  void *h, *y;
  float* scales;
  int rows, d;
  int wbf16;
  int vec;       // every row of x, res, h, y and w starts on 16 bytes (y: 8 for e4m3)
  float eps;
};

// Element (i, j) of a thread's VPT groups of 8: 8 neighbours where vectors can be used,
// else one every `nt` elements, so that a warp's loads stay together.
__device__ __forceinline__ int elem(bool vec, int i, int j, int t, int nt) {
  return vec ? (t + i * nt) * 8 + j : (i * 8 + j) * nt + t;
}

template <typename T>
__device__ __forceinline__ void row_load(const T* p, bool vec, int i, int t, int nt, int d, float (&v)[8]) {
  const int e0 = elem(true, i, 0, t, nt);
  if (vec && e0 + 8 <= d) {
    load8(p + e0, v);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int e = elem(vec, i, j, t, nt);
    v[j] = e < d ? to_f32(p[e]) : 0.f;
  }
}

template <typename T>
__device__ __forceinline__ void row_store(T* p, bool vec, int i, int t, int nt, int d, const float (&v)[8]) {
  const int e0 = elem(true, i, 0, t, nt);
  if (vec && e0 + 8 <= d) {
    store8(p + e0, v);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int e = elem(vec, i, j, t, nt);
    if (e < d) p[e] = from_f32<T>(v[j]);
  }
}

__device__ __forceinline__ uint8_t e4m3(float v) {
  return (uint8_t)__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3);
}

__device__ __forceinline__ void row_store_e4m3(uint8_t* p, bool vec, int i, int t, int nt, int d,
                                               const float (&v)[8]) {
  const int e0 = elem(true, i, 0, t, nt);
  if (vec && e0 + 8 <= d) {
    uint32_t q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      q[j] = __nv_cvt_float2_to_fp8x2(make_float2(v[2 * j], v[2 * j + 1]), __NV_SATFINITE, __NV_E4M3);
    *reinterpret_cast<uint2*>(p + e0) = make_uint2(q[0] | (q[1] << 16), q[2] | (q[3] << 16));
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int e = elem(vec, i, j, t, nt);
    if (e < d) p[e] = e4m3(v[j]);
  }
}

__device__ __forceinline__ void load_w(const NormParams& P, int i, int t, int nt, float (&v)[8]) {
  if (P.wbf16)
    row_load((const __nv_bfloat16*)P.w, P.vec, i, t, nt, P.d, v);
  else
    row_load((const float*)P.w, P.vec, i, t, nt, P.d, v);
}

// A row's scale, and its values over it: a product with the reciprocal, or a quotient
// where the scale is so small that the reciprocal would overflow.
struct RowScale {
  float s, inv;
  bool small;
  __device__ explicit RowScale(float amax) {
    s = amax / E4M3_MAX;
    if (s == 0.f) s = 1.f;
    small = s < FLT_MIN;
    inv = 1.f / s;
  }
  __device__ __forceinline__ float operator()(float y) const { return small ? y / s : y * inv; }
};

// One row per CTA, VPT groups of 8 elements per thread in registers.
template <typename T, bool E4M3, int VPT>
__global__ void __launch_bounds__(1024) k_rmsnorm(const NormParams P) {
  __shared__ float slots[2][32];
  const int t = threadIdx.x, nt = blockDim.x;
  const int64_t row = blockIdx.x;
  const T* x = (const T*)P.x + row * P.ldx;
  const T* res = P.res ? (const T*)P.res + row * P.ldr : nullptr;
  float h[VPT][8];
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    row_load(x, P.vec, i, t, nt, P.d, h[i]);
    if (res) {
      float r[8];
      row_load(res, P.vec, i, t, nt, P.d, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i][j] += r[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = fmaf(h[i][j], h[i][j], ss);
  }
  if (P.h) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) row_store((T*)P.h + row * P.ldh, P.vec, i, t, nt, P.d, h[i]);
  }
  ss = cta_all(ss, AddOp(), slots[0]);
  const float rho = 1.f / sqrtf(ss / (float)P.d + P.eps);
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    float w[8];
    load_w(P, i, t, nt, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      h[i][j] = h[i][j] * rho * w[j];
      if (E4M3) amax = max_nan(amax, fabsf(h[i][j]));
    }
    if (!E4M3) row_store((T*)P.y + row * P.ldy, P.vec, i, t, nt, P.d, h[i]);
  }
  if constexpr (E4M3) {
    const RowScale sc(cta_all(amax, MaxNanOp(), slots[1]));
    if (t == 0) P.scales[row] = sc.s;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i][j] = sc(h[i][j]);
      row_store_e4m3((uint8_t*)P.y + row * P.ldy, P.vec, i, t, nt, P.d, h[i]);
    }
  }
}

// Rows too long for registers: x and r are read again for y (and for its maximum).
// h may be x or r, so it is written last, in the pass that forms y.
template <typename T, bool E4M3>
__global__ void __launch_bounds__(1024) k_rmsnorm_long(const NormParams P) {
  __shared__ float slots[2][32];
  const int64_t row = blockIdx.x;
  const T* x = (const T*)P.x + row * P.ldx;
  const T* res = P.res ? (const T*)P.res + row * P.ldr : nullptr;
  auto at = [&](int e) { return res ? to_f32(x[e]) + to_f32(res[e]) : to_f32(x[e]); };
  auto weight = [&](int e) {
    return P.wbf16 ? to_f32(((const __nv_bfloat16*)P.w)[e]) : ((const float*)P.w)[e];
  };
  float ss = 0.f;
  for (int e = threadIdx.x; e < P.d; e += blockDim.x) {
    const float v = at(e);
    ss = fmaf(v, v, ss);
  }
  ss = cta_all(ss, AddOp(), slots[0]);
  const float rho = 1.f / sqrtf(ss / (float)P.d + P.eps);
  float amax = 0.f;
  if (E4M3) {
    for (int e = threadIdx.x; e < P.d; e += blockDim.x)
      amax = max_nan(amax, fabsf(at(e) * rho * weight(e)));
    amax = cta_all(amax, MaxNanOp(), slots[1]);
  }
  const RowScale sc(amax);
  if (E4M3 && threadIdx.x == 0) P.scales[row] = sc.s;
  for (int e = threadIdx.x; e < P.d; e += blockDim.x) {
    const float v = at(e), y = v * rho * weight(e);
    if (P.h) ((T*)P.h + row * P.ldh)[e] = from_f32<T>(v);
    if constexpr (E4M3)
      ((uint8_t*)P.y + row * P.ldy)[e] = e4m3(sc(y));
    else
      ((T*)P.y + row * P.ldy)[e] = from_f32<T>(y);
  }
}

struct NormBackParams {
  const void *dy, *h, *w, *dsum;
  int64_t lddy, ldh, ldds, lddx;
  void* dx;
  float *rho, *part;   // [rows]; [parts][d]
  int rows, d, wbf16, parts;
  float eps;
};

// dx of a row, and its rho for the weight's gradient.
template <typename T>
__global__ void __launch_bounds__(256) k_rmsnorm_dx(const NormBackParams P) {
  __shared__ float slots[2][32];
  const int64_t row = blockIdx.x;
  const T* h = (const T*)P.h + row * P.ldh;
  const T* dy = (const T*)P.dy + row * P.lddy;
  auto weight = [&](int e) {
    return P.wbf16 ? to_f32(((const __nv_bfloat16*)P.w)[e]) : ((const float*)P.w)[e];
  };
  float ss = 0.f, c = 0.f;
  for (int e = threadIdx.x; e < P.d; e += blockDim.x) {
    const float v = to_f32(h[e]);
    ss = fmaf(v, v, ss);
    c = fmaf(weight(e) * to_f32(dy[e]), v, c);
  }
  ss = cta_all(ss, AddOp(), slots[0]);
  c = cta_all(c, AddOp(), slots[1]) / (float)P.d;
  const float rho = 1.f / sqrtf(ss / (float)P.d + P.eps), k = rho * rho * c;
  if (threadIdx.x == 0) P.rho[row] = rho;
  for (int e = threadIdx.x; e < P.d; e += blockDim.x) {
    float v = rho * (weight(e) * to_f32(dy[e]) - to_f32(h[e]) * k);
    if (P.dsum) v += to_f32(((const T*)P.dsum + row * P.ldds)[e]);
    ((T*)P.dx + row * P.lddx)[e] = from_f32<T>(v);
  }
}

// Columns of part p: dy h rho over the rows p, p + parts, ...
template <typename T>
__global__ void __launch_bounds__(256) k_rmsnorm_dw(const NormBackParams P) {
  const int e = blockIdx.x * blockDim.x + threadIdx.x;
  if (e >= P.d) return;
  float s = 0.f;
  for (int64_t row = blockIdx.y; row < P.rows; row += P.parts)
    s = fmaf(to_f32(((const T*)P.dy + row * P.lddy)[e]) * to_f32(((const T*)P.h + row * P.ldh)[e]),
             P.rho[row], s);
  P.part[(int64_t)blockIdx.y * P.d + e] = s;
}

// dw = the parts' sum, always in the same order: 32 columns a CTA, 32 ranges of parts.
__global__ void __launch_bounds__(1024) k_sum_parts(const float* part, int parts, int d, float* dw) {
  __shared__ float s[32][33];
  const int c = blockIdx.x * 32 + threadIdx.x;
  float v = 0.f;
  if (c < d)
    for (int p = threadIdx.y; p < parts; p += 32) v += part[(int64_t)p * d + c];
  s[threadIdx.y][threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.y == 0 && c < d) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) t += s[i][threadIdx.x];
    dw[c] = t;
  }
}

// Rows share their parts of dw among this many CTAs.
int back_parts(int rows) { return std::min(rows, 4 * ROW_SMS); }

template <typename T, bool E4M3>
int norm_launch(const NormParams& P, cudaStream_t s) {
  const int groups = ceil_div(P.d, 8);
  if (groups > 2 * 1024) {
    k_rmsnorm_long<T, E4M3><<<P.rows, 1024, 0, s>>>(P);
  } else if (groups <= 1024) {
    k_rmsnorm<T, E4M3, 1><<<P.rows, (unsigned)round_up(groups, 32), 0, s>>>(P);
  } else {
    k_rmsnorm<T, E4M3, 2><<<P.rows, (unsigned)round_up(ceil_div(groups, 2), 32), 0, s>>>(P);
  }
  BK_CUDA_OK(cudaGetLastError());
  return BAKRON_OK;
}

bool float_dtype(int t) { return t == BAKRON_F32 || t == BAKRON_BF16; }

}  // namespace
}  // namespace bakron

using namespace bakron;

extern "C" int bakron_rmsnorm(const void* x, int dtype, int rows, int d, int64_t ldx,
                              const void* residual, int64_t ldr, const void* weight, int wdtype,
                              float eps, void* sum, int64_t lds, void* y, int ydtype, int64_t ldy,
                              float* scales, void* stream) {
  if (rows < 0 || d < 1 || d > NORM_MAX_D || !float_dtype(dtype) || !float_dtype(wdtype) ||
      (ydtype != dtype && ydtype != BAKRON_E4M3) || !(eps >= 0.f))
    return BAKRON_ERR_INVALID_ARG;
  if (rows == 0) return BAKRON_OK;
  if (!x || !weight || !y || ldx < d || ldy < d || (residual && ldr < d) || (sum && lds < d) ||
      (ydtype == BAKRON_E4M3 && !scales))
    return BAKRON_ERR_INVALID_ARG;
  const int es = dtype == BAKRON_F32 ? 4 : 2;
  const bool q = ydtype == BAKRON_E4M3;
  NormParams P{};
  P.x = x; P.res = residual; P.w = weight; P.h = sum; P.y = y; P.scales = scales;
  P.ldx = ldx; P.ldr = ldr; P.ldh = lds; P.ldy = ldy;
  P.rows = rows; P.d = d; P.wbf16 = wdtype == BAKRON_BF16; P.eps = eps;
  P.vec = aligned16(x, ldx * es) && (!residual || aligned16(residual, ldr * es)) &&
          (!sum || aligned16(sum, lds * es)) && aligned16(weight, 0) &&
          (q ? ((uintptr_t)y | (uintptr_t)ldy) % 8 == 0 : aligned16(y, ldy * es));
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == BAKRON_F32) return q ? norm_launch<float, true>(P, s) : norm_launch<float, false>(P, s);
  return q ? norm_launch<__nv_bfloat16, true>(P, s) : norm_launch<__nv_bfloat16, false>(P, s);
}

extern "C" size_t bakron_rmsnorm_backward_workspace_bytes(int rows, int d) {
  if (rows < 0 || d < 1 || d > NORM_MAX_D) return 0;
  return align256((size_t)rows * 4) + (size_t)back_parts(rows) * d * 4 + 256;
}

extern "C" int bakron_rmsnorm_backward(const void* dy, int64_t lddy, const void* h, int64_t ldh,
                                       int dtype, int rows, int d, const void* weight, int wdtype,
                                       float eps, const void* dsum, int64_t ldds, void* dx,
                                       int64_t lddx, float* dw, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  if (rows < 0 || d < 1 || d > NORM_MAX_D || !float_dtype(dtype) || !float_dtype(wdtype) ||
      !(eps >= 0.f) || !dw || !workspace)
    return BAKRON_ERR_INVALID_ARG;
  if (rows > 0 && (!dy || !h || !weight || !dx || lddy < d || ldh < d || lddx < d || (dsum && ldds < d)))
    return BAKRON_ERR_INVALID_ARG;
  if (workspace_bytes < bakron_rmsnorm_backward_workspace_bytes(rows, d)) return BAKRON_ERR_WORKSPACE;
  cudaStream_t s = (cudaStream_t)stream;
  NormBackParams P{};
  P.dy = dy; P.h = h; P.w = weight; P.dsum = dsum; P.dx = dx;
  P.lddy = lddy; P.ldh = ldh; P.ldds = ldds; P.lddx = lddx;
  P.rows = rows; P.d = d; P.wbf16 = wdtype == BAKRON_BF16; P.parts = back_parts(rows); P.eps = eps;
  P.rho = (float*)workspace;
  P.part = (float*)((char*)workspace + align256((size_t)rows * 4));
  if (rows > 0) {
    const dim3 gw((unsigned)ceil_div(d, 256), (unsigned)P.parts);
    if (dtype == BAKRON_F32) {
      k_rmsnorm_dx<float><<<rows, 256, 0, s>>>(P);
      k_rmsnorm_dw<float><<<gw, 256, 0, s>>>(P);
    } else {
      k_rmsnorm_dx<__nv_bfloat16><<<rows, 256, 0, s>>>(P);
      k_rmsnorm_dw<__nv_bfloat16><<<gw, 256, 0, s>>>(P);
    }
    BK_CUDA_OK(cudaGetLastError());
  }
  k_sum_parts<<<(unsigned)ceil_div(d, 32), dim3(32, 32), 0, s>>>(P.part, P.parts, d, dw);
  BK_CUDA_OK(cudaGetLastError());
  return BAKRON_OK;
}
