// bakron_rmsnorm and bakron_rmsnorm_backward.
//
//   h = x + r,  rho = 1 / sqrt(mean(h^2) + eps),  y = w h rho
//   dx = rho (w dy - h rho^2 mean(w dy h)) + dsum,  dw = sum over rows of dy h rho
//
// The sum h is formed and kept in fp32; it is rounded once where it is stored, and y
// comes from the unrounded one.
#include <algorithm>

#include "norm.cuh"

namespace bakron {
namespace {

struct NormParams {
  const void *x, *res, *w;
  int64_t ldx, ldr, ldh, ldy;
  void *h, *y;
  float* scales;
  int rows, d;
  int wbf16;
  int vec;       // d % 8 is 0, and every row of x, res, h, y and w starts on 16 bytes (y: 8 for e4m3)
  float eps;
};

// VPT groups of 8 elements of a row per thread in registers.  Bound by memory: what counts is
// that loads stay in flight.  Long rows (AHEAD): a CTA takes the rows blockIdx.x,
// + gridDim.x, ..., with the next one on its way while this one is summed and written
// (16381 x 8192 bf16 with a residual 178 us, 6.0 TB/s; a row per CTA 197).  Shorter ones: a row
// per CTA, with fewer registers and more CTAs at once (16384 x 1000 bf16 24 us, ahead 45).
template <typename T, bool E4M3, int VPT, bool AHEAD, bool VEC>
__global__ void __launch_bounds__(AHEAD || VPT > 1 ? 512 : 1024, AHEAD && VPT * sizeof(T) <= 4 ? 2 : 1)
    k_rmsnorm(const NormParams P) {
  __shared__ float slots[2][2][32];
  const int t = threadIdx.x, nt = blockDim.x;
  struct Row {
    Raw8<T> x[VPT], r[VPT];
  };
  auto load_row = [&](int64_t row, Row& o) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      raw_load<VEC>((const T*)P.x + row * P.ldx, i, t, nt, P.d, o.x[i]);
      if (P.res) raw_load<VEC>((const T*)P.res + row * P.ldr, i, t, nt, P.d, o.r[i]);
    }
  };
  Row next;
  if (blockIdx.x < P.rows) load_row(blockIdx.x, next);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < P.rows; row += gridDim.x, turn ^= 1) {
    float h[VPT][8];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      next.x[i].get(h[i]);
      if (P.res) {
        float r[8];
        next.r[i].get(r);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] += r[j];
      }
    }
    if (AHEAD && row + gridDim.x < P.rows) load_row(row + gridDim.x, next);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fmaf(h[i][j], h[i][j], ss);
      if (P.h) row_store<VEC>((T*)P.h + row * P.ldh, i, t, nt, P.d, h[i]);
    }
    ss = cta_all(ss, AddOp(), slots[turn][0]);
    const float rho = 1.f / sqrtf(ss / (float)P.d + P.eps);
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float w[8];
      load_w<VEC>(P.w, P.wbf16, i, t, nt, P.d, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[i][j] = h[i][j] * rho * w[j];
        if (E4M3) amax = max_nan(amax, fabsf(h[i][j]));
      }
      if (!E4M3) row_store<VEC>((T*)P.y + row * P.ldy, i, t, nt, P.d, h[i]);
    }
    if constexpr (E4M3) {
      const RowScale sc(cta_all(amax, MaxNanOp(), slots[turn][1]));
      if (t == 0) P.scales[row] = sc.s;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] = sc(h[i][j]);
        row_store_e4m3<VEC>((uint8_t*)P.y + row * P.ldy, i, t, nt, P.d, h[i]);
      }
    }
    if (!AHEAD) break;
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
  int vec;             // as for the norm
  float eps;
};

// A CTA takes the rows blockIdx.x, + gridDim.x, ...: each is read once while its two sums are
// formed and used again for dx; the weight's gradient stays in registers from row to row
// and leaves as one part per CTA.  Four groups of 8 a thread: what a row costs beside its
// elements (two sums over the CTA, addresses, rho) is shared by 32 of them (with 8 a
// thread the kernel was bound by instructions).  Rows that vectors can be used for wait in a
// ring of RING rows in shared memory, copied there without registers, so that loads stay
// in flight: 8192 x 4096 in bf16 with dsum 47 us, held in registers (RING 0) 69.
constexpr int BACK_VPT = 4;

template <typename T, typename W, bool VEC, int RING, int MAXT>
__global__ void __launch_bounds__(MAXT) k_rmsnorm_back(const NormBackParams P) {
  constexpr int VPT = BACK_VPT;
  constexpr bool HOLD = sizeof(T) == 2 && RING == 0;      // dsum too
  // The rings leave little of the SM's memory to its cache: the weight stays in registers.
  constexpr bool KEEP_W = RING > 0 && MAXT == 256;
  static_assert(VEC || RING == 0, "whole vectors");
  __shared__ float2 slots[2][16];
  extern __shared__ __align__(16) unsigned char nb_ring[];   // [RING][h, dy, dsum][d]
  const int t = threadIdx.x, nt = blockDim.x, warp = t >> 5, lane = t & 31, warps = nt >> 5;
  pdl_trigger();      // the parts' sum may get ready; it waits for this grid's end
  Raw8<W> weight[KEEP_W ? VPT : 1];
  if constexpr (KEEP_W) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) raw_load<VEC>((const W*)P.w, i, t, nt, P.d, weight[i]);
  }
  auto get_w = [&](int i, float (&w)[8]) {
    if constexpr (KEEP_W)
      weight[i].get(w);
    else
      row_load<VEC>((const W*)P.w, i, t, nt, P.d, w);
  };
  float dw[VPT][8] = {};
  int turn = 0, slot = 0;
  T* ring = reinterpret_cast<T*>(nb_ring);
  auto fetch = [&](int64_t row, int to) {      // each thread its own groups
    if (row < P.rows) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int e0 = elem<true>(i, 0, t, nt);
        if (e0 >= P.d) continue;
        T* at = ring + (int64_t)to * 3 * P.d + e0;
#pragma unroll
        for (int k = 0; k < 8; k += 16 / (int)sizeof(T)) {
          copy16(at + k, (const T*)P.h + row * P.ldh + e0 + k);
          copy16(at + P.d + k, (const T*)P.dy + row * P.lddy + e0 + k);
          if (P.dsum) copy16(at + 2 * P.d + k, (const T*)P.dsum + row * P.ldds + e0 + k);
        }
      }
    }
    copies_group();
  };
  if constexpr (RING > 0) {
#pragma unroll
    for (int s = 0; s < RING - 1; ++s) fetch(blockIdx.x + (int64_t)s * gridDim.x, s);
  }
  for (int64_t row = blockIdx.x; row < P.rows; row += gridDim.x, turn ^= 1) {
    Raw8<T> h[RING ? 1 : VPT], dy[RING ? 1 : VPT], ds[HOLD ? VPT : 1];
    const T* here = ring + (int64_t)slot * 3 * P.d;
    if constexpr (RING > 0) {
      copies_left<(RING > 1 ? RING - 2 : 0)>();
      fetch(row + (int64_t)(RING - 1) * gridDim.x, slot == 0 ? RING - 1 : slot - 1);
      slot = slot == RING - 1 ? 0 : slot + 1;
    } else {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        raw_load<VEC>((const T*)P.h + row * P.ldh, i, t, nt, P.d, h[i]);
        raw_load<VEC>((const T*)P.dy + row * P.lddy, i, t, nt, P.d, dy[i]);
        if (HOLD && P.dsum) raw_load<VEC>((const T*)P.dsum + row * P.ldds, i, t, nt, P.d, ds[HOLD ? i : 0]);
      }
    }
    auto get = [&](int i, float (&a)[8], float (&b)[8]) {
      if constexpr (RING > 0) {
        row_load<true>(here, i, t, nt, P.d, a);
        row_load<true>(here + P.d, i, t, nt, P.d, b);
      } else {
        h[i].get(a);
        dy[i].get(b);
      }
    };
    float ss = 0.f, c = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float a[8], b[8], w[8];
      get(i, a, b);
      get_w(i, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ss = fmaf(a[j], a[j], ss);
        c = fmaf(w[j] * b[j], a[j], c);
      }
    }
    // both sums in one butterfly: the lower half warp goes on with ss, the upper with c
    const bool up = lane & 16;
    float v = (up ? c : ss) + __shfl_xor_sync(0xffffffffu, up ? ss : c, 16);
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((lane & 15) == 0) (up ? slots[turn][warp].y : slots[turn][warp].x) = v;
    if (warps > 1)
      __syncthreads();      // (the other turn's slots were read before this)
    else
      __syncwarp();
    ss = c = 0.f;
    for (int w = 0; w < warps; ++w) {
      const float2 s = slots[turn][w];
      ss += s.x;
      c += s.y;
    }
    const float rho = 1.f / sqrtf(ss / (float)P.d + P.eps), k = rho * rho * (c / (float)P.d);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float a[8], b[8], w[8], o[8];
      get(i, a, b);
      get_w(i, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dw[i][j] = fmaf(b[j] * a[j], rho, dw[i][j]);
        o[j] = fmaf(rho, w[j] * b[j], -(rho * k) * a[j]);
      }
      if (P.dsum) {
        if (HOLD)
          ds[HOLD ? i : 0].get(a);
        else if (RING > 0)
          row_load<true>(here + 2 * P.d, i, t, nt, P.d, a);
        else
          row_load<VEC>((const T*)P.dsum + row * P.ldds, i, t, nt, P.d, a);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] += a[j];
      }
      row_store<VEC>((T*)P.dx + row * P.lddx, i, t, nt, P.d, o);
    }
  }
  float* part = P.part + (int64_t)blockIdx.x * P.d;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = elem<VEC>(i, j, t, nt);
      if (e < P.d) part[e] = dw[i][j];
    }
}

// Rows too long for that: dx of a row, and its rho for the weight's gradient.
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

// Threads of a CTA (0: rows too long), and CTAs, each with its part of dw: what an SM holds.
constexpr int NB_SMEM = 220 * 1024;      // of an SM's, beside each CTA's kilobyte
int back_threads(int d) {
  const int nt = (int)round_up(ceil_div(ceil_div(d, 8), BACK_VPT), 32);
  return nt <= 512 ? nt : 0;
}
struct BackPlan {
  int ring, ctas;      // rows of the ring, CTAs of an SM
  BackPlan(int d, int es, bool vec) {
    const int nt = back_threads(d), row = 3 * d * es;
    ring = !nt || !vec || 2 * row > NB_SMEM ? 0 : nt > 256 || 2 * 3 * row > NB_SMEM ? 2 : 3;
    ctas = nt ? std::max(1, 512 / nt) : 4;
    // (one CTA fits wherever its ring does: NB_SMEM leaves 8 KB of the SM's)
    if (ring) ctas = std::max(1, std::min(640 / nt, NB_SMEM / (ring * row + 1024)));
  }
};
int back_parts(int rows, int d, int es, bool vec) {
  return std::min(rows, ROW_SMS * BackPlan(d, es, vec).ctas);
}

template <typename K>
cudaError_t back_attr(K kernel) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, NB_SMEM);
}

template <typename T, typename W>
cudaError_t back_launch(const NormBackParams& P, cudaStream_t s) {
  const int nt = back_threads(P.d), ring = BackPlan(P.d, sizeof(T), P.vec).ring;
  if (!nt) {
    k_rmsnorm_dx<T><<<P.rows, 256, 0, s>>>(P);
    k_rmsnorm_dw<T><<<dim3((unsigned)ceil_div(P.d, 256), (unsigned)P.parts), 256, 0, s>>>(P);
    return cudaGetLastError();
  }
  static OncePerDevice once;
  const cudaError_t e = once([] {
    cudaError_t a = back_attr(k_rmsnorm_back<T, W, true, 2, 256>);
    if (a == cudaSuccess) a = back_attr(k_rmsnorm_back<T, W, true, 3, 256>);
    if (a == cudaSuccess) a = back_attr(k_rmsnorm_back<T, W, true, 2, 512>);
    return a;
  });
  if (e != cudaSuccess) return e;
  const auto kernel = ring == 0  ? (P.vec ? k_rmsnorm_back<T, W, true, 0, 512> : k_rmsnorm_back<T, W, false, 0, 512>)
                      : nt > 256 ? k_rmsnorm_back<T, W, true, 2, 512>
                      : ring == 2 ? k_rmsnorm_back<T, W, true, 2, 256> : k_rmsnorm_back<T, W, true, 3, 256>;
  kernel<<<P.parts, nt, (size_t)ring * 3 * P.d * sizeof(T), s>>>(P);
  return cudaGetLastError();
}

template <typename T, bool E4M3, bool VEC>
int norm_launch(const NormParams& P, cudaStream_t s) {
  const int groups = ceil_div(P.d, 8);
  const bool many = P.rows > 2 * ROW_SMS;
  if (groups > 2048) {
    k_rmsnorm_long<T, E4M3><<<P.rows, 1024, 0, s>>>(P);
  } else if (groups > 1024 || (many && groups > 512)) {
    const int vpt = groups > 1024 ? 4 : 2, nt = (int)round_up(ceil_div(groups, vpt), 32);
    const int ctas = std::min(P.rows, ROW_SMS * ((vpt * (int)sizeof(T) <= 4 ? 1024 : 512) / nt));
    if (vpt == 4)
      k_rmsnorm<T, E4M3, 4, true, VEC><<<ctas, nt, 0, s>>>(P);
    else
      k_rmsnorm<T, E4M3, 2, true, VEC><<<ctas, nt, 0, s>>>(P);
  } else if (many && groups > 256) {
    k_rmsnorm<T, E4M3, 2, false, VEC><<<P.rows, (unsigned)round_up(ceil_div(groups, 2), 32), 0, s>>>(P);
  } else {
    k_rmsnorm<T, E4M3, 1, false, VEC><<<P.rows, (unsigned)round_up(groups, 32), 0, s>>>(P);
  }
  BK_CUDA_OK(cudaGetLastError());
  return BAKRON_OK;
}

template <typename T>
int norm_kinds(const NormParams& P, bool q, cudaStream_t s) {
  if (q) return P.vec ? norm_launch<T, true, true>(P, s) : norm_launch<T, true, false>(P, s);
  return P.vec ? norm_launch<T, false, true>(P, s) : norm_launch<T, false, false>(P, s);
}

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
  P.vec = d % 8 == 0 && aligned16(x, ldx * es) && (!residual || aligned16(residual, ldr * es)) &&
          (!sum || aligned16(sum, lds * es)) && aligned16(weight, 0) &&
          (q ? ((uintptr_t)y | (uintptr_t)ldy) % 8 == 0 : aligned16(y, ldy * es));
  cudaStream_t s = (cudaStream_t)stream;
  return dtype == BAKRON_F32 ? norm_kinds<float>(P, q, s) : norm_kinds<__nv_bfloat16>(P, q, s);
}

extern "C" size_t bakron_rmsnorm_backward_workspace_bytes(int rows, int d) {
  if (rows < 0 || d < 1 || d > NORM_MAX_D) return 0;
  int parts = 0;      // whichever way the call goes
  for (int es : {2, 4})
    for (bool vec : {false, true}) parts = std::max(parts, back_parts(rows, d, es, vec));
  return align256((size_t)rows * 4) + (size_t)parts * d * 4 + 256;
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
  P.rows = rows; P.d = d; P.wbf16 = wdtype == BAKRON_BF16; P.eps = eps;
  P.rho = (float*)workspace;
  P.part = (float*)((char*)workspace + align256((size_t)rows * 4));
  if (rows > 0) {
    const int es = dtype == BAKRON_F32 ? 4 : 2;
    P.vec = d % 8 == 0 && aligned16(dy, lddy * es) && aligned16(h, ldh * es) && (!dsum || aligned16(dsum, ldds * es)) &&
            aligned16(dx, lddx * es) && aligned16(weight, 0);
    P.parts = back_parts(rows, d, es, P.vec);
    const auto launch = dtype == BAKRON_F32 ? (P.wbf16 ? back_launch<float, __nv_bfloat16> : back_launch<float, float>)
                                            : (P.wbf16 ? back_launch<__nv_bfloat16, __nv_bfloat16>
                                                       : back_launch<__nv_bfloat16, float>);
    BK_CUDA_OK(launch(P, s));
  }
  BK_CUDA_OK(launch_pdl(k_sum_parts, dim3((unsigned)ceil_div(d, 32)), dim3(32, 32), 0, s, P.part, P.parts, d, dw,
                       (float*)nullptr));
  return BAKRON_OK;
}
