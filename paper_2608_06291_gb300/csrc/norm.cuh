// What the two norms (norm.cu, layernorm.cu) share: a row's elements in a CTA's registers, the
// 8-bit results' scale, and the sum of the weights' gradients.
#pragma once

#include <float.h>

#include "rowops.cuh"

namespace bakron {

constexpr int NORM_MAX_D = 1 << 16;
constexpr float E4M3_MAX = 448.f;

// Element (i, j) of a thread's VPT groups of 8: 8 neighbours where vectors can be used (VEC:
// d is a multiple of 8 and every row starts on 16 bytes), else one every `nt` elements, so
// that a warp's loads stay together.
template <bool VEC>
__device__ __forceinline__ int elem(int i, int j, int t, int nt) {
  return VEC ? (t + i * nt) * 8 + j : (i * 8 + j) * nt + t;
}

template <bool VEC, typename T>
__device__ __forceinline__ void row_load(const T* p, int i, int t, int nt, int d, float (&v)[8]) {
  if constexpr (VEC) {
    const int e0 = elem<true>(i, 0, t, nt);
    if (e0 < d) {
      load8(p + e0, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = elem<false>(i, j, t, nt);
      v[j] = e < d ? to_f32(p[e]) : 0.f;
    }
  }
}

template <bool VEC, typename T>
__device__ __forceinline__ void row_store(T* p, int i, int t, int nt, int d, const float (&v)[8]) {
  if constexpr (VEC) {
    const int e0 = elem<true>(i, 0, t, nt);
    if (e0 < d) store8(p + e0, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = elem<false>(i, j, t, nt);
      if (e < d) p[e] = from_f32<T>(v[j]);
    }
  }
}

__device__ __forceinline__ uint8_t e4m3(float v) {
  return (uint8_t)__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3);
}

template <bool VEC>
__device__ __forceinline__ void row_store_e4m3(uint8_t* p, int i, int t, int nt, int d, const float (&v)[8]) {
  if constexpr (VEC) {
    const int e0 = elem<true>(i, 0, t, nt);
    if (e0 >= d) return;
    uint32_t q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      q[j] = __nv_cvt_float2_to_fp8x2(make_float2(v[2 * j], v[2 * j + 1]), __NV_SATFINITE, __NV_E4M3);
    *reinterpret_cast<uint2*>(p + e0) = make_uint2(q[0] | (q[1] << 16), q[2] | (q[3] << 16));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = elem<false>(i, j, t, nt);
      if (e < d) p[e] = e4m3(v[j]);
    }
  }
}

// 8 elements as they are stored.
template <typename T>
struct Raw8;
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    a = make_float4(v[0], v[1], v[2], v[3]);
    b = make_float4(v[4], v[5], v[6], v[7]);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};
template <>
struct Raw8<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    a = make_uint4(bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]), bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7]));
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
    v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z); v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
  }
};

template <bool VEC, typename T>
__device__ __forceinline__ void raw_load(const T* p, int i, int t, int nt, int d, Raw8<T>& r) {
  if (VEC && elem<true>(i, 0, t, nt) < d) {
    r.load(p + elem<true>(i, 0, t, nt));
  } else {
    float v[8];
    if constexpr (VEC) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.f;
    } else {
      row_load<false>(p, i, t, nt, d, v);
    }
    r.set(v);
  }
}

// The weight, fp32 or bf16.
template <bool VEC>
__device__ __forceinline__ void load_w(const void* w, int bf16, int i, int t, int nt, int d, float (&v)[8]) {
  if (bf16)
    row_load<VEC>((const __nv_bfloat16*)w, i, t, nt, d, v);
  else
    row_load<VEC>((const float*)w, i, t, nt, d, v);
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

// dw = the parts' sum, always in the same order: 32 columns a CTA, 32 ranges of parts, whose
// sums a warp joins pairwise (one after another they were the largest part of dw's error).
// blockIdx.y: which of a part's rows of d, and of the results.
static __global__ void __launch_bounds__(1024) k_sum_parts(const float* part, int parts, int d, float* out0, float* out1) {
  __shared__ float s[32][33];
  const int c = blockIdx.x * 32 + threadIdx.x;
  pdl_wait();
  float v = 0.f;
  if (c < d)
    for (int p = threadIdx.y; p < parts; p += 32) v += part[((int64_t)p * gridDim.y + blockIdx.y) * d + c];
  s[threadIdx.y][threadIdx.x] = v;
  __syncthreads();
  v = warp_all(s[threadIdx.x][threadIdx.y], AddOp());
  const int at = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && at < d) (blockIdx.y ? out1 : out0)[at] = v;
}

inline bool float_dtype(int t) { return t == BAKRON_F32 || t == BAKRON_BF16; }

}  // namespace bakron
