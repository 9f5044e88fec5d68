// bakron_layernorm and bakron_layernorm_backward.
//
//   h = x + r,  mu = mean(h),  rho = 1 / sqrt(mean((h - mu)^2) + eps),  y = w (h - mu) rho + b
//   g = w dy,  c = h - mu
//   dx = rho (g - mean(g) - c rho^2 mean(g c)) + dsum
//   dw = sum over rows of dy c rho,  db = sum over rows of dy
//
// The mean first, then the sums of what is left of each element (not mean(h^2) - mu^2, which
// loses the variance of rows far from zero): a row stays where the second pass finds it, in
// registers or shared memory.  h is formed and kept in fp32 and rounded once where it is
// stored; y comes from the unrounded one.
#include <algorithm>

#include "norm.cuh"

namespace bakron {
namespace {

struct LayerParams {
  const void *x, *res, *w, *b;
  int64_t ldx, ldr, ldh, ldy;
  void *h, *y;
  float* scales;
  int rows, d;
  int wbf16, bbf16;
  int vec;       // d % 8 is 0, and every row of x, res, h, y, w and b starts on 16 bytes (y: 8 for e4m3)
  float eps;
};

// Of a group's 8 elements, those inside the row.
template <bool VEC>
__device__ __forceinline__ bool inside(int i, int j, int t, int nt, int d) {
  return VEC ? elem<true>(i, 0, t, nt) < d : elem<false>(i, j, t, nt) < d;
}

// VPT groups of 8 elements of a row per thread in registers, bound by memory; AHEAD as in the
// root-mean-square norm: long rows, a CTA takes several with the next one on its way.  16381 x 8192 bf16 with a
// residual 173 us (6.2 TB/s); 1 x 4096 to e4m3 4.8.
template <typename T, bool E4M3, int VPT, bool AHEAD, bool VEC>
__global__ void __launch_bounds__(AHEAD || VPT > 1 ? 512 : 1024, AHEAD && VPT * sizeof(T) <= 4 ? 2 : 1)
    k_layernorm(const LayerParams P) {
  __shared__ float slots[2][3][32];
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
    float sum = 0.f;
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
      for (int j = 0; j < 8; ++j) sum += h[i][j];
      if (P.h) row_store<VEC>((T*)P.h + row * P.ldh, i, t, nt, P.d, h[i]);
    }
    const float mu = cta_all(sum, AddOp(), slots[turn][0]) / (float)P.d;
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[i][j] = inside<VEC>(i, j, t, nt, P.d) ? h[i][j] - mu : 0.f;      // (0 - mu) rho may be infinite
        ss = fmaf(h[i][j], h[i][j], ss);
      }
    ss = cta_all(ss, AddOp(), slots[turn][1]);
    const float rho = 1.f / sqrtf(ss / (float)P.d + P.eps);
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float w[8], b[8] = {};
      load_w<VEC>(P.w, P.wbf16, i, t, nt, P.d, w);
      if (P.b) load_w<VEC>(P.b, P.bbf16, i, t, nt, P.d, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[i][j] = fmaf(h[i][j] * rho, w[j], b[j]);      // (w and b are 0 past the row)
        if (E4M3) amax = max_nan(amax, fabsf(h[i][j]));
      }
      if (!E4M3) row_store<VEC>((T*)P.y + row * P.ldy, i, t, nt, P.d, h[i]);
    }
    if constexpr (E4M3) {
      const RowScale sc(cta_all(amax, MaxNanOp(), slots[turn][2]));
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

// Rows too long for registers: x and r are read again in each pass.  h may be x or r, so it is
// written last, in the pass that forms y.
template <typename T, bool E4M3>
__global__ void __launch_bounds__(1024) k_layernorm_long(const LayerParams P) {
  __shared__ float slots[3][32];
  const int64_t row = blockIdx.x;
  const T* x = (const T*)P.x + row * P.ldx;
  const T* res = P.res ? (const T*)P.res + row * P.ldr : nullptr;
  auto at = [&](int e) { return res ? to_f32(x[e]) + to_f32(res[e]) : to_f32(x[e]); };
  auto param = [](const void* p, int bf16, int e) { return bf16 ? to_f32(((const __nv_bfloat16*)p)[e]) : ((const float*)p)[e]; };
  float sum = 0.f, ss = 0.f;
  for (int e = threadIdx.x; e < P.d; e += blockDim.x) sum += at(e);
  const float mu = cta_all(sum, AddOp(), slots[0]) / (float)P.d;
  for (int e = threadIdx.x; e < P.d; e += blockDim.x) {
    const float c = at(e) - mu;
    ss = fmaf(c, c, ss);
  }
  ss = cta_all(ss, AddOp(), slots[1]);
  const float rho = 1.f / sqrtf(ss / (float)P.d + P.eps);
  auto norm = [&](float v, int e) { return fmaf((v - mu) * rho, param(P.w, P.wbf16, e), P.b ? param(P.b, P.bbf16, e) : 0.f); };
  float amax = 0.f;
  if (E4M3) {
    for (int e = threadIdx.x; e < P.d; e += blockDim.x) amax = max_nan(amax, fabsf(norm(at(e), e)));
    amax = cta_all(amax, MaxNanOp(), slots[2]);
  }
  const RowScale sc(amax);
  if (E4M3 && threadIdx.x == 0) P.scales[row] = sc.s;
  for (int e = threadIdx.x; e < P.d; e += blockDim.x) {
    const float v = at(e), y = norm(v, e);
    if (P.h) ((T*)P.h + row * P.ldh)[e] = from_f32<T>(v);
    if constexpr (E4M3)
      ((uint8_t*)P.y + row * P.ldy)[e] = e4m3(sc(y));
    else
      ((T*)P.y + row * P.ldy)[e] = from_f32<T>(y);
  }
}

struct LayerBackParams {
  const void *dy, *h, *w, *dsum;
  int64_t lddy, ldh, ldds, lddx;
  void* dx;
  float *stats, *part;   // [rows][mu, rho]; [parts][dw, db][d]
  int rows, d, wbf16, parts;
  int vec;               // as for the norm
  float eps;
};

// Two sums over the CTA (at most 32 warps) in one butterfly: the lower half warp goes on with a, the
// upper with b, in the warp and then over the warps.
struct TwoSlots {
  float v[2][32];
};
__device__ __forceinline__ void two_all(float& a, float& b, TwoSlots& slots) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int up = lane >> 4, in = lane & 15;
  float v = (up ? b : a) + __shfl_xor_sync(0xffffffffu, up ? a : b, 16);
#pragma unroll
  for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (warps > 1) {
    if (in == 0) slots.v[up][warp] = v;
    __syncthreads();
    v = in < warps ? slots.v[up][in] : 0.f;
    if (in + 16 < warps) v += slots.v[up][in + 16];
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  }
  a = __shfl_sync(0xffffffffu, v, 0);
  b = __shfl_sync(0xffffffffu, v, 16);
}

// A CTA takes the rows blockIdx.x, + gridDim.x, ...; both parameters' gradients stay in registers
// from row to row and leave as one part per CTA.
//
// Many rows of up to 8192 elements that vectors can be used for: 16 elements a thread, read once
// from a ring of RING rows that vector copies fill ahead, and kept in fp32, as pairs, through the three
// passes (mean, sums of what is left, dx).  What bounds it is latency, with 16 warps an SM, as the registers allow
// (issue slots 54% busy, DRAM 58%): 8192 x 4096 in bf16 with dsum takes 56 us with the parts' sum, and with the
// row read back from shared memory and widened in each pass, one value an instruction, took 98.
constexpr int LB_GROUPS = 1024;      // groups of 8: 512 threads
template <typename T, typename W, int RING, int MAXT>
__global__ void __launch_bounds__(MAXT, 512 / MAXT) k_layernorm_back(const LayerBackParams P) {
  __shared__ TwoSlots slots[2];
  extern __shared__ __align__(16) unsigned char lb_ring[];   // [RING][h, dy, dsum][d]
  const int t = threadIdx.x, nt = blockDim.x;
  auto pairs = [](const float (&v)[8], Two* p) {
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = Two(v[2 * j], v[2 * j + 1]);
  };
  const Two zero(0.f, 0.f);
  Two w[8], dw[8], db[8];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float v[8];
    row_load<true>((const W*)P.w, i, t, nt, P.d, v);
    pairs(v, w + 4 * i);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) dw[j] = db[j] = zero;
  T* ring = reinterpret_cast<T*>(lb_ring);
  auto fetch = [&](int64_t row, int to) {      // each thread its own groups
    T* at = ring + (int64_t)to * 3 * P.d;
    if (row < P.rows) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int e0 = elem<true>(i, 0, t, nt);
        if (e0 >= P.d) continue;
#pragma unroll
        for (int k = 0; k < 8; k += 16 / (int)sizeof(T)) {
          copy16(at + e0 + k, (const T*)P.h + row * P.ldh + e0 + k);
          copy16(at + P.d + e0 + k, (const T*)P.dy + row * P.lddy + e0 + k);
          if (P.dsum) copy16(at + 2 * P.d + e0 + k, (const T*)P.dsum + row * P.ldds + e0 + k);
        }
      }
    }
    copies_group();
  };
#pragma unroll
  for (int s = 0; s < RING - 1; ++s) fetch(blockIdx.x + (int64_t)s * gridDim.x, s);
  const float inv = 1.f / (float)P.d;
  int slot = 0;
  for (int64_t row = blockIdx.x; row < P.rows; row += gridDim.x) {
    const T* here = ring + (int64_t)slot * 3 * P.d;
    copies_left<RING - 2>();
    fetch(row + (int64_t)(RING - 1) * gridDim.x, slot == 0 ? RING - 1 : slot - 1);
    slot = slot == RING - 1 ? 0 : slot + 1;
    Two c[8], b[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float v[8];
      row_load<true>(here, i, t, nt, P.d, v);
      pairs(v, c + 4 * i);
      row_load<true>(here + P.d, i, t, nt, P.d, v);
      pairs(v, b + 4 * i);
    }
    Two s0 = c[0], s1 = Two::mul(w[0], b[0]);
#pragma unroll
    for (int j = 1; j < 8; ++j) {
      s0 = Two::add(s0, c[j]);
      s1 = Two::fma(w[j], b[j], s1);
    }
    float mu, mg, ss, gc, hi;
    s0.get(mu, hi);
    mu += hi;
    s1.get(mg, hi);
    mg += hi;
    two_all(mu, mg, slots[0]);
    mu /= (float)P.d;      // as the norm has it: a product with 1 / d may miss a constant row's value
    mg *= inv;
    const Two minus_mu(-mu, -mu);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool in = elem<true>(i, 0, t, nt) < P.d;
#pragma unroll
      for (int j = 4 * i; j < 4 * i + 4; ++j) c[j] = in ? Two::add(c[j], minus_mu) : zero;
    }
    s0 = Two::mul(c[0], c[0]);
    s1 = Two::mul(Two::mul(w[0], b[0]), c[0]);
#pragma unroll
    for (int j = 1; j < 8; ++j) {
      s0 = Two::fma(c[j], c[j], s0);
      s1 = Two::fma(Two::mul(w[j], b[j]), c[j], s1);
    }
    s0.get(ss, hi);
    ss += hi;
    s1.get(gc, hi);
    gc += hi;
    two_all(ss, gc, slots[1]);
    const float rho = 1.f / sqrtf(ss * inv + P.eps), k = rho * rho * (gc * inv);
    const Two rr(rho, rho), minus_k(-k, -k), minus_mg(-mg, -mg);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float o[8];
#pragma unroll
      for (int j = 4 * i; j < 4 * i + 4; ++j) {
        dw[j] = Two::fma(Two::mul(b[j], c[j]), rr, dw[j]);
        db[j] = Two::add(db[j], b[j]);
        const Two v = Two::mul(rr, Two::fma(minus_k, c[j], Two::fma(w[j], b[j], minus_mg)));
        v.get(o[2 * (j & 3)], o[2 * (j & 3) + 1]);
      }
      if (P.dsum) {
        float v[8];
        row_load<true>(here + 2 * P.d, i, t, nt, P.d, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] += v[j];
      }
      row_store<true>((T*)P.dx + row * P.lddx, i, t, nt, P.d, o);
    }
  }
  pdl_trigger();
  float* part = P.part + (int64_t)blockIdx.x * 2 * P.d;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float v[8], u[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      dw[4 * i + j].get(v[2 * j], v[2 * j + 1]);
      db[4 * i + j].get(u[2 * j], u[2 * j + 1]);
    }
    row_store<true>(part, i, t, nt, P.d, v);
    row_store<true>(part + P.d, i, t, nt, P.d, u);
  }
}

// Longer rows, and rows that vectors cannot be used for: up to 1024 threads, so 64 registers.  A row is
// read three times from shared memory, and a thread reads back only what it put there; a ring where
// vectors can be used (with the weight in registers: it leaves little of the SM's memory to its cache),
// else a row (RING 1) is copied when its turn comes.
template <typename T, typename W, bool VEC, int RING, int VPT>
__global__ void __launch_bounds__(1024) k_layernorm_back_wide(const LayerBackParams P) {
  constexpr bool KEEP_W = RING > 1;
  static_assert(VEC || RING == 1, "whole vectors");
  __shared__ TwoSlots slots[2];
  extern __shared__ __align__(16) unsigned char lb_ring[];   // [RING][h, dy, dsum][d]
  const int t = threadIdx.x, nt = blockDim.x;
  pdl_trigger();      // the parts' sum may get ready; it waits for this grid's end
  float dw[VPT][8] = {}, db[VPT][8] = {};
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
  int slot = 0;
  T* ring = reinterpret_cast<T*>(lb_ring);
  auto fetch = [&](int64_t row, int to) {      // each thread its own groups
    T* at = ring + (int64_t)to * 3 * P.d;
    if (row < P.rows) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        if constexpr (VEC) {
          const int e0 = elem<true>(i, 0, t, nt);
          if (e0 >= P.d) continue;
#pragma unroll
          for (int k = 0; k < 8; k += 16 / (int)sizeof(T)) {
            copy16(at + e0 + k, (const T*)P.h + row * P.ldh + e0 + k);
            copy16(at + P.d + e0 + k, (const T*)P.dy + row * P.lddy + e0 + k);
            if (P.dsum) copy16(at + 2 * P.d + e0 + k, (const T*)P.dsum + row * P.ldds + e0 + k);
          }
        } else {
          Raw8<T> a, b;
          raw_load<false>((const T*)P.h + row * P.ldh, i, t, nt, P.d, a);
          raw_load<false>((const T*)P.dy + row * P.lddy, i, t, nt, P.d, b);
          float u[8], v[8];
          a.get(u);
          b.get(v);
          row_store<false>(at, i, t, nt, P.d, u);
          row_store<false>(at + P.d, i, t, nt, P.d, v);
        }
      }
    }
    if (VEC) copies_group();
  };
  if constexpr (VEC) {
#pragma unroll
    for (int s = 0; s < RING - 1; ++s) fetch(blockIdx.x + (int64_t)s * gridDim.x, s);
  }
  const float inv = 1.f / (float)P.d;
  for (int64_t row = blockIdx.x; row < P.rows; row += gridDim.x) {
    const T* here = ring + (int64_t)slot * 3 * P.d;
    if constexpr (VEC && RING == 1) {
      fetch(row, 0);
      copies_left<0>();
    } else if constexpr (VEC) {
      copies_left<RING - 2>();
      fetch(row + (int64_t)(RING - 1) * gridDim.x, slot == 0 ? RING - 1 : slot - 1);
      slot = slot == RING - 1 ? 0 : slot + 1;
    } else {
      fetch(row, 0);
    }
    float mu = 0.f, mg = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float a[8], b[8], w[8];
      row_load<VEC>(here, i, t, nt, P.d, a);
      row_load<VEC>(here + P.d, i, t, nt, P.d, b);
      get_w(i, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        mu += a[j];
        mg = fmaf(w[j], b[j], mg);
      }
    }
    two_all(mu, mg, slots[0]);
    mu /= (float)P.d;      // as the norm has it: a product with 1 / d may miss a constant row's value
    mg *= inv;
    float ss = 0.f, gc = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float a[8], b[8], w[8];
      row_load<VEC>(here, i, t, nt, P.d, a);
      row_load<VEC>(here + P.d, i, t, nt, P.d, b);
      get_w(i, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float c = inside<VEC>(i, j, t, nt, P.d) ? a[j] - mu : 0.f;
        ss = fmaf(c, c, ss);
        gc = fmaf(w[j] * b[j], c, gc);
      }
    }
    two_all(ss, gc, slots[1]);
    const float rho = 1.f / sqrtf(ss * inv + P.eps), k = rho * rho * (gc * inv);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float a[8], b[8], w[8], o[8];
      row_load<VEC>(here, i, t, nt, P.d, a);
      row_load<VEC>(here + P.d, i, t, nt, P.d, b);
      get_w(i, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float c = a[j] - mu;
        dw[i][j] = fmaf(b[j] * c, rho, dw[i][j]);      // (dy is 0 past the row)
        db[i][j] += b[j];
        o[j] = rho * fmaf(-k, c, fmaf(w[j], b[j], -mg));
      }
      if (P.dsum) {
        row_load<VEC>(VEC ? here + 2 * P.d : (const T*)P.dsum + row * P.ldds, i, t, nt, P.d, a);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] += a[j];
      }
      row_store<VEC>((T*)P.dx + row * P.lddx, i, t, nt, P.d, o);
    }
  }
  float* part = P.part + (int64_t)blockIdx.x * 2 * P.d;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = elem<VEC>(i, j, t, nt);
      if (e < P.d) {
        part[e] = dw[i][j];
        part[P.d + e] = db[i][j];
      }
    }
}

template <typename T>
__device__ __forceinline__ void load_n(const T* p, float (&v)[1]) { v[0] = to_f32(*p); }
template <typename T>
__device__ __forceinline__ void load_n(const T* p, float (&v)[8]) { load8(p, v); }

// dx of a row, and its mean and rho for the parameters' gradients: rows too long for that, and few
// rows, where what counts is to start early and to run short loops (the kernel above unrolls 16
// elements three times; executed once, its instructions come from memory: 37 x 11003 in fp32 40 us).
template <typename T, bool VEC>
__global__ void __launch_bounds__(1024) k_layernorm_dx(const LayerBackParams P) {
  constexpr int N = VEC ? 8 : 1;
  __shared__ TwoSlots slots[2];
  const int64_t row = blockIdx.x;
  const T* h = (const T*)P.h + row * P.ldh;
  const T* dy = (const T*)P.dy + row * P.lddy;
  auto grad = [&](int e, float (&g)[N]) {
    float w[N];
    load_n(dy + e, g);
    if (P.wbf16)
      load_n((const __nv_bfloat16*)P.w + e, w);
    else
      load_n((const float*)P.w + e, w);
#pragma unroll
    for (int j = 0; j < N; ++j) g[j] *= w[j];
  };
  const float inv = 1.f / (float)P.d;
  const int step = blockDim.x * N;
  float mu = 0.f, mg = 0.f, ss = 0.f, gc = 0.f;
#pragma unroll 4
  for (int e = threadIdx.x * N; e < P.d; e += step) {
    float a[N], g[N];
    load_n(h + e, a);
    grad(e, g);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      mu += a[j];
      mg += g[j];
    }
  }
  two_all(mu, mg, slots[0]);
  mu /= (float)P.d;      // as the norm has it
  mg *= inv;
#pragma unroll 4
  for (int e = threadIdx.x * N; e < P.d; e += step) {
    float a[N], g[N];
    load_n(h + e, a);
    grad(e, g);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float c = a[j] - mu;
      ss = fmaf(c, c, ss);
      gc = fmaf(g[j], c, gc);
    }
  }
  two_all(ss, gc, slots[1]);
  pdl_trigger();
  const float rho = 1.f / sqrtf(ss * inv + P.eps), k = rho * rho * (gc * inv);
  if (threadIdx.x == 0) {
    P.stats[2 * row] = mu;
    P.stats[2 * row + 1] = rho;
  }
#pragma unroll 4
  for (int e = threadIdx.x * N; e < P.d; e += step) {
    float a[N], g[N];
    load_n(h + e, a);
    grad(e, g);
#pragma unroll
    for (int j = 0; j < N; ++j) g[j] = rho * fmaf(-k, a[j] - mu, g[j] - mg);
    if (P.dsum) {
      load_n((const T*)P.dsum + row * P.ldds + e, a);
#pragma unroll
      for (int j = 0; j < N; ++j) g[j] += a[j];
    }
    if constexpr (VEC)
      store8((T*)P.dx + row * P.lddx + e, g);
    else
      ((T*)P.dx + row * P.lddx)[e] = from_f32<T>(g[0]);
  }
}

// Few rows: dw and db from the rows themselves, joined as k_sum_parts joins parts.
template <typename T>
__global__ void __launch_bounds__(1024) k_layernorm_sums(const LayerBackParams P, float* dw, float* db) {
  __shared__ float s[2][32][33];
  const int c = blockIdx.x * 32 + threadIdx.x;
  pdl_wait();
  float v = 0.f, b = 0.f;
  if (c < P.d)
    for (int64_t row = threadIdx.y; row < P.rows; row += 32) {
      const float dy = to_f32(((const T*)P.dy + row * P.lddy)[c]);
      v = fmaf(dy * (to_f32(((const T*)P.h + row * P.ldh)[c]) - P.stats[2 * row]), P.stats[2 * row + 1], v);
      b += dy;
    }
  s[0][threadIdx.y][threadIdx.x] = v;
  s[1][threadIdx.y][threadIdx.x] = b;
  __syncthreads();
  v = warp_all(s[0][threadIdx.x][threadIdx.y], AddOp());
  b = warp_all(s[1][threadIdx.x][threadIdx.y], AddOp());
  const int at = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && at < P.d) {
    dw[at] = v;
    db[at] = b;
  }
}

// Columns of part p: dy c rho and dy over the rows p, p + parts, ...
template <typename T>
__global__ void __launch_bounds__(256) k_layernorm_dwb(const LayerBackParams P) {
  const int e = blockIdx.x * blockDim.x + threadIdx.x;
  if (e >= P.d) return;
  float s = 0.f, b = 0.f;
  for (int64_t row = blockIdx.y; row < P.rows; row += P.parts) {
    const float dy = to_f32(((const T*)P.dy + row * P.lddy)[e]);
    s = fmaf(dy * (to_f32(((const T*)P.h + row * P.ldh)[e]) - P.stats[2 * row]), P.stats[2 * row + 1], s);
    b += dy;
  }
  P.part[(int64_t)blockIdx.y * 2 * P.d + e] = s;
  P.part[((int64_t)blockIdx.y * 2 + 1) * P.d + e] = b;
}

// The launch: groups of 8 a thread (0: dx by itself), threads, rows of the ring, CTAs an SM.
constexpr int LB_SMEM = 220 * 1024;      // of an SM, with a kilobyte and the slots beside each ring
constexpr int LB_FEW = 4 * ROW_SMS;      // rows: up to here, no loop over them (600 x 4096 bf16 15.6 us, with one 17.7; 1000 24.4, 21.4)
struct LayerPlan {
  bool few, paired;
  int vpt, nt, ring, ctas;
  LayerPlan(int rows, int d, int es, bool vec) {
    const int groups = ceil_div(d, 8), row = 3 * d * es;
    few = rows <= LB_FEW;
    ring = 1;
    vpt = few || groups > 2048 ? 0 : groups > 1024 ? 2 : 1;
    if (vpt && vec && 2 * row <= LB_SMEM) vpt = ring = 2;
    paired = ring == 2 && groups <= LB_GROUPS;
    nt = vpt ? (int)round_up(ceil_div(groups, vpt), 32) : few ? (int)std::min<int64_t>(1024, round_up(vec ? groups : ceil_div(d, 4), 32)) : 256;
    ctas = vpt ? std::max(1, std::min((paired ? 512 : 1024) / nt, LB_SMEM / (ring * row + 1536))) : 4;
    while (ring > 1 && ring < (paired ? 4 : 2) && ctas * ((ring + 1) * row + 1536) <= LB_SMEM) ++ring;
  }
  int parts(int rows) const { return few ? 0 : std::min(rows, ROW_SMS * ctas); }
};

template <typename T, typename W>
cudaError_t layer_back_launch(const LayerBackParams& P, const LayerPlan& L, cudaStream_t s) {
  if (!L.vpt) {
    if (P.vec)
      k_layernorm_dx<T, true><<<P.rows, L.nt, 0, s>>>(P);
    else
      k_layernorm_dx<T, false><<<P.rows, L.nt, 0, s>>>(P);
    if (!L.few) k_layernorm_dwb<T><<<dim3((unsigned)ceil_div(P.d, 256), (unsigned)P.parts), 256, 0, s>>>(P);
    return cudaGetLastError();
  }
  static OncePerDevice once;
  const cudaError_t e = once([] {
    cudaError_t a = cudaSuccess;
    for (auto k : {k_layernorm_back<T, W, 2, 256>, k_layernorm_back<T, W, 3, 256>, k_layernorm_back<T, W, 4, 256>,
                   k_layernorm_back<T, W, 2, 512>, k_layernorm_back<T, W, 3, 512>, k_layernorm_back<T, W, 4, 512>,
                   k_layernorm_back_wide<T, W, false, 1, 1>, k_layernorm_back_wide<T, W, false, 1, 2>,
                   k_layernorm_back_wide<T, W, true, 1, 2>, k_layernorm_back_wide<T, W, true, 2, 2>})
      if (a == cudaSuccess) a = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, LB_SMEM);
    return a;
  });
  if (e != cudaSuccess) return e;
  auto kernel = L.ring == 2 ? k_layernorm_back_wide<T, W, true, 2, 2>
                            : k_layernorm_back_wide<T, W, true, 1, 2>;      // fp32 rows so long that a ring holds one
  if (!P.vec)
    kernel = L.vpt == 1 ? k_layernorm_back_wide<T, W, false, 1, 1> : k_layernorm_back_wide<T, W, false, 1, 2>;
  else if (L.paired && L.nt <= 256)
    kernel = L.ring == 2   ? k_layernorm_back<T, W, 2, 256>
             : L.ring == 3 ? k_layernorm_back<T, W, 3, 256> : k_layernorm_back<T, W, 4, 256>;
  else if (L.paired)
    kernel = L.ring == 2   ? k_layernorm_back<T, W, 2, 512>
             : L.ring == 3 ? k_layernorm_back<T, W, 3, 512> : k_layernorm_back<T, W, 4, 512>;
  kernel<<<P.parts, L.nt, (size_t)L.ring * 3 * P.d * sizeof(T), s>>>(P);
  return cudaGetLastError();
}

template <typename T, bool E4M3, bool VEC>
int layer_launch(const LayerParams& P, cudaStream_t s) {
  const int groups = ceil_div(P.d, 8);
  const bool many = P.rows > 2 * ROW_SMS;
  if (groups > 2048) {
    k_layernorm_long<T, E4M3><<<P.rows, 1024, 0, s>>>(P);
  } else if (groups > 1024 || (many && groups > 512)) {
    const int vpt = groups > 1024 ? 4 : 2, nt = (int)round_up(ceil_div(groups, vpt), 32);
    const int ctas = std::min(P.rows, ROW_SMS * ((vpt * (int)sizeof(T) <= 4 ? 1024 : 512) / nt));
    if (vpt == 4)
      k_layernorm<T, E4M3, 4, true, VEC><<<ctas, nt, 0, s>>>(P);
    else
      k_layernorm<T, E4M3, 2, true, VEC><<<ctas, nt, 0, s>>>(P);
  } else if (many && groups > 256) {
    k_layernorm<T, E4M3, 2, false, VEC><<<P.rows, (unsigned)round_up(ceil_div(groups, 2), 32), 0, s>>>(P);
  } else {
    k_layernorm<T, E4M3, 1, false, VEC><<<P.rows, (unsigned)round_up(groups, 32), 0, s>>>(P);
  }
  BK_CUDA_OK(cudaGetLastError());
  return BAKRON_OK;
}

template <typename T>
int layer_kinds(const LayerParams& P, bool q, cudaStream_t s) {
  if (q) return P.vec ? layer_launch<T, true, true>(P, s) : layer_launch<T, true, false>(P, s);
  return P.vec ? layer_launch<T, false, true>(P, s) : layer_launch<T, false, false>(P, s);
}

}  // namespace
}  // namespace bakron

using namespace bakron;

extern "C" int bakron_layernorm(const void* x, int dtype, int rows, int d, int64_t ldx, const void* residual,
                                int64_t ldr, const void* weight, int wdtype, const void* bias, int bdtype, float eps,
                                void* sum, int64_t lds, void* y, int ydtype, int64_t ldy, float* scales, void* stream) {
  if (rows < 0 || d < 1 || d > NORM_MAX_D || !float_dtype(dtype) || !float_dtype(wdtype) ||
      (bias && !float_dtype(bdtype)) || (ydtype != dtype && ydtype != BAKRON_E4M3) || !(eps >= 0.f))
    return BAKRON_ERR_INVALID_ARG;
  if (rows == 0) return BAKRON_OK;
  if (!x || !weight || !y || ldx < d || ldy < d || (residual && ldr < d) || (sum && lds < d) ||
      (ydtype == BAKRON_E4M3 && !scales))
    return BAKRON_ERR_INVALID_ARG;
  const int es = dtype == BAKRON_F32 ? 4 : 2;
  const bool q = ydtype == BAKRON_E4M3;
  LayerParams P{};
  P.x = x; P.res = residual; P.w = weight; P.b = bias; P.h = sum; P.y = y; P.scales = scales;
  P.ldx = ldx; P.ldr = ldr; P.ldh = lds; P.ldy = ldy;
  P.rows = rows; P.d = d; P.wbf16 = wdtype == BAKRON_BF16; P.bbf16 = bdtype == BAKRON_BF16; P.eps = eps;
  P.vec = d % 8 == 0 && aligned16(x, ldx * es) && (!residual || aligned16(residual, ldr * es)) &&
          (!sum || aligned16(sum, lds * es)) && aligned16(weight, 0) && aligned16(bias, 0) &&
          (q ? ((uintptr_t)y | (uintptr_t)ldy) % 8 == 0 : aligned16(y, ldy * es));
  cudaStream_t s = (cudaStream_t)stream;
  return dtype == BAKRON_F32 ? layer_kinds<float>(P, q, s) : layer_kinds<__nv_bfloat16>(P, q, s);
}

extern "C" size_t bakron_layernorm_backward_workspace_bytes(int rows, int d) {
  if (rows < 0 || d < 1 || d > NORM_MAX_D) return 0;
  int parts = 0;      // whichever way the call goes
  for (int es : {2, 4})
    for (bool vec : {false, true}) parts = std::max(parts, LayerPlan(rows, d, es, vec).parts(rows));
  return align256((size_t)rows * 8) + (size_t)parts * d * 8 + 256;
}

extern "C" int bakron_layernorm_backward(const void* dy, int64_t lddy, const void* h, int64_t ldh, int dtype, int rows,
                                         int d, const void* weight, int wdtype, float eps, const void* dsum,
                                         int64_t ldds, void* dx, int64_t lddx, float* dw, float* db, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  if (rows < 0 || d < 1 || d > NORM_MAX_D || !float_dtype(dtype) || !float_dtype(wdtype) || !(eps >= 0.f) || !dw ||
      !db || !workspace || (uintptr_t)workspace % 16 != 0)
    return BAKRON_ERR_INVALID_ARG;
  if (rows > 0 && (!dy || !h || !weight || !dx || lddy < d || ldh < d || lddx < d || (dsum && ldds < d)))
    return BAKRON_ERR_INVALID_ARG;
  if (workspace_bytes < bakron_layernorm_backward_workspace_bytes(rows, d)) return BAKRON_ERR_WORKSPACE;
  cudaStream_t s = (cudaStream_t)stream;
  LayerBackParams P{};
  P.dy = dy; P.h = h; P.w = weight; P.dsum = dsum; P.dx = dx;
  P.lddy = lddy; P.ldh = ldh; P.ldds = ldds; P.lddx = lddx;
  P.rows = rows; P.d = d; P.wbf16 = wdtype == BAKRON_BF16; P.eps = eps;
  P.stats = (float*)workspace;
  P.part = (float*)((char*)workspace + align256((size_t)rows * 8));
  if (rows > 0) {
    const int es = dtype == BAKRON_F32 ? 4 : 2;
    P.vec = d % 8 == 0 && aligned16(dy, lddy * es) && aligned16(h, ldh * es) && (!dsum || aligned16(dsum, ldds * es)) &&
            aligned16(dx, lddx * es) && aligned16(weight, 0);
    const LayerPlan L(rows, d, es, P.vec);
    P.parts = L.parts(rows);
    const auto launch = dtype == BAKRON_F32
                            ? (P.wbf16 ? layer_back_launch<float, __nv_bfloat16> : layer_back_launch<float, float>)
                            : (P.wbf16 ? layer_back_launch<__nv_bfloat16, __nv_bfloat16>
                                       : layer_back_launch<__nv_bfloat16, float>);
    BK_CUDA_OK(launch(P, L, s));
  }
  if (rows > 0 && rows <= LB_FEW)
    BK_CUDA_OK(launch_pdl(dtype == BAKRON_F32 ? k_layernorm_sums<float> : k_layernorm_sums<__nv_bfloat16>,
                          dim3((unsigned)ceil_div(d, 32)), dim3(32, 32), 0, s, P, dw, db));
  else
    BK_CUDA_OK(launch_pdl(k_sum_parts, dim3((unsigned)ceil_div(d, 32), 2), dim3(32, 32), 0, s, P.part, P.parts, d, dw, db));
  return BAKRON_OK;
}
