// bakron_token_logprobs and bakron_token_logprobs_backward.
//
//   lse = m + log(sum exp(l - m)),  logp = l[target] - lse,  H = lse - sum p l
//   dl_j = g ([j = target] - p_j) - u p_j (log p_j + H)
//
// Forward: one pass.  A row is cut into tiles of 1024 elements; the warps of a row take them
// in turn.  Each lane keeps s = sum 2^t and u = sum 2^t t, t = l log2(e) - m, m the running
// maximum rounded up to a whole number (so that changing it only moves exponents), and
// joins them at the end (warp, CTA, cluster): lse = (m + log2 s) ln 2, H = (log2 s - u / s) ln 2.
// Each warp keeps its 32 best (value, index), one a lane, and looks at a tile's elements
// only where a lane's maximum, which it has anyway, beats the last one that counts.
// What bounds it: memory without a list (4095 x 128256 bf16: 162 us, 6.5 TB/s); with one, the
// dependent steps of its first insertions (top 20: 214 us, 4.9 TB/s).  In fp32 (1024 rows)
// 84 and 101 us.  The gradient is bound by memory: 4096 x 128256 bf16 324 us, 6.5 TB/s.
//
// t in one fused operation errs by 2^-25 |l|, so rows whose maximum is beyond +-1024 are
// gone through once more with l - max, which is exact where it matters (k_logprob's end).
#include <cooperative_groups.h>
#include <limits.h>

#include <algorithm>

#include "rowops.cuh"

namespace cg = cooperative_groups;

namespace bakron {
namespace {

constexpr int TOP_MAX = 32;
constexpr int V_MAX = INT_MAX - 1023;  // an index, or a row's end rounded up to a tile, passes no 32 bits
constexpr float LSE_EXACT = 1024.f;   // up to here lse's rounding is below 2^-14
constexpr float LOG2E = 1.4426950408889634f;
constexpr double LN2 = 0.6931471805599453;
constexpr float FAR = -1000.f;        // exp() of it is 0; finite, so that 0 * FAR is 0
constexpr float USUAL = 1024.f;       // row maxima up to here, either sign, take the one pass
constexpr float NOTHING = -2048.f;    // values below it are 0 beside any usual maximum
constexpr int LP_WARPS = 16;          // most warps of a CTA
constexpr int LP_LANE = 32;           // elements of a tile per lane
constexpr int LP_TILE = 32 * LP_LANE;
constexpr int LP_STAGES = 3;          // tiles of a warp in shared memory: one used, two on their way

__device__ __forceinline__ float exp2_fast(float v) {   // 2 ulp, results below 2^-126 are 0
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

struct LogprobParams {
  const void* logits;
  int64_t ld;
  const int64_t* targets;
  int rows, v, top;
  float *logp, *entropy, *lse, *top_logp;
  int* top_ids;
};

// The larger value first, the lower index first among equal ones.
__device__ __forceinline__ bool before(float a, int i, float b, int j) {
  return a > b || (a == b && i < j);
}

// m, s, u of some elements; join() makes them those of both sets.  NaNs stay in s and u.
struct Sums {
  float m, s, u;
  __device__ __forceinline__ void to(float to_m) {   // to_m >= m
    const float dm = m == to_m ? 0.f : fmaxf(m - to_m, FAR), f = exp2_fast(dm);
    u = f * fmaf(dm, s, u);
    s *= f;
    m = to_m;
  }
  __device__ __forceinline__ void join(Sums o) {
    const float top = fmaxf(m, o.m);
    to(top);
    o.to(top);
    s += o.s;
    u += o.u;
  }
  __device__ __forceinline__ void join_warp() {
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      Sums b;
      b.m = __shfl_xor_sync(0xffffffffu, m, d);
      b.s = __shfl_xor_sync(0xffffffffu, s, d);
      b.u = __shfl_xor_sync(0xffffffffu, u, d);
      join(b);
    }
  }
};

// A row as aligned 16-byte vectors of PER elements: vector 0 starts `off` elements before
// the row.
template <typename T>
struct RowVectors {
  static constexpr int PER = 16 / sizeof(T);
  const T* row;
  const uint4* base;
  int off, v, last;   // vectors 1 .. last - 1 lie inside the row, and 0 if off is 0
  __device__ RowVectors(const T* r, int n) : row(r), v(n) {
    off = (int)(((uintptr_t)r & 15) / sizeof(T));
    base = reinterpret_cast<const uint4*>((uintptr_t)r & ~(uintptr_t)15);
    last = (int)(((int64_t)off + n) / PER);
  }
  __device__ __forceinline__ int count() const { return (int)(((int64_t)off + v + PER - 1) / PER); }
  __device__ __forceinline__ bool inside(int i) const { return i < last && (i > 0 || off == 0); }
  __device__ __forceinline__ int64_t first(int i) const { return (int64_t)i * PER - off; }
};

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  __nv_bfloat162 r = __hmax2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<uint32_t*>(&r);
}

// A lane's 32 elements of a tile, as loaded: U vectors, 32 apart.
template <typename T>
struct Tile {
  static constexpr int PER = 16 / sizeof(T), U = LP_LANE / PER;
  uint4 r[U];
  // The tile's vectors on their way to `to` (32 * U of them, each lane its own); -inf beside the row.
  __device__ __forceinline__ static void fetch(const RowVectors<T>& R, int tile, int lane, uint4* to) {
    const int v0 = tile * 32 * U;
    if (R.inside(v0) && v0 + 32 * U <= R.last) {     // uniform: the whole tile
#pragma unroll
      for (int u = 0; u < U; ++u) copy16(to + u * 32 + lane, R.base + v0 + u * 32 + lane);
      return;
    }
#pragma unroll 1
    for (int u = 0; u < U; ++u) {
      const int i = v0 + u * 32 + lane;
      if (R.inside(i)) {
        copy16(to + u * 32 + lane, R.base + i);
        continue;
      }
      T* o = reinterpret_cast<T*>(to + u * 32 + lane);
      const int64_t e0 = R.first(i);
#pragma unroll
      for (int j = 0; j < PER; ++j)
        o[j] = e0 + j >= 0 && e0 + j < R.v ? R.row[e0 + j] : from_f32<T>(-INFINITY);
    }
  }
  __device__ __forceinline__ void read(const uint4* from, int lane) {
#pragma unroll
    for (int u = 0; u < U; ++u) r[u] = from[u * 32 + lane];
  }
  __device__ __forceinline__ float max() const {   // of what is no NaN, where there is any
    if constexpr (sizeof(T) == 2) {
      uint32_t m = max_bf16x2(max_bf16x2(r[0].x, r[0].y), max_bf16x2(r[0].z, r[0].w));
#pragma unroll
      for (int u = 1; u < U; ++u)
        m = max_bf16x2(m, max_bf16x2(max_bf16x2(r[u].x, r[u].y), max_bf16x2(r[u].z, r[u].w)));
      return fmaxf(bf16_lo(m), bf16_hi(m));
    } else {
      float m = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u)
        m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(r[u].x), __uint_as_float(r[u].y)),
                           fmaxf(__uint_as_float(r[u].z), __uint_as_float(r[u].w))));
      return m;
    }
  }
  // Adds the elements: 2^t and 2^t t, pairwise.  -inf (and what is as good as it) is cut to
  // a finite value, for the product's sake.
  __device__ __forceinline__ void add(Sums& a) const {
    const float m = a.m == -INFINITY ? 0.f : a.m;
    const Two k(LOG2E, LOG2E), nm(-m, -m);
    Two s(0.f, 0.f), u(0.f, 0.f);
    auto two = [&](float x, float y) {
      const Two t = Two::fma(Two(x, y), k, nm);
      t.get(x, y);
      const Two e(exp2_fast(x), exp2_fast(y));
      s = Two::add(s, e);
      u = Two::fma(e, t, u);
    };
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const uint32_t w[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t c;
          asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(w[j]), "r"(0xFE96FE96u));   // -1e38
          two(bf16_lo(c), bf16_hi(c));
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; j += 2)
          two(max_nan(__uint_as_float(w[j]), -1e38f), max_nan(__uint_as_float(w[j + 1]), -1e38f));
      }
    }
    float x, y;
    s.get(x, y);
    a.s += x + y;
    u.get(x, y);
    a.u += x + y;
  }
};

// The 32 best of a warp, best first, one a lane; `at` is the last one that counts.
struct TopList {
  float v = -INFINITY, at_v = -INFINITY;
  int i = INT_MAX, at_i = INT_MAX;
  __device__ __forceinline__ void insert(float x, int xi, int lane, int top) {
    const int pos = __popc(__ballot_sync(0xffffffffu, before(v, i, x, xi)));
    const float pv = __shfl_up_sync(0xffffffffu, v, 1);
    const int pi = __shfl_up_sync(0xffffffffu, i, 1);
    if (lane >= pos) {
      v = lane == pos ? x : pv;
      i = lane == pos ? xi : pi;
    }
    at_v = __shfl_sync(0xffffffffu, v, top - 1);
    at_i = __shfl_sync(0xffffffffu, i, top - 1);
  }
  // The 32 best of this list and another, (ov, oi) of the lane's place in it.
  __device__ __forceinline__ void merge(float ov, int oi, int lane) {
    ov = __shfl_sync(0xffffffffu, ov, 31 - lane);
    oi = __shfl_sync(0xffffffffu, oi, 31 - lane);
    if (before(ov, oi, v, i)) {
      v = ov;
      i = oi;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const float pv = __shfl_xor_sync(0xffffffffu, v, o);
      const int pi = __shfl_xor_sync(0xffffffffu, i, o);
      if (before(pv, pi, v, i) == ((lane & o) == 0)) {
        v = pv;
        i = pi;
      }
    }
  }
};

// The n-th largest of the lanes' values (n = 1..32), no NaN among them.
__device__ __forceinline__ float nth_largest(float v, int n, int lane) {
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int o = k >> 1; o; o >>= 1) {
      const float p = __shfl_xor_sync(0xffffffffu, v, o);
      const bool up = ((lane & o) == 0) == ((lane & k) == 0 || k == 32);
      v = up ? fmaxf(v, p) : fminf(v, p);
    }
  return __shfl_sync(0xffffffffu, v, n - 1);
}

// What a warp knows of its part of a row, for the ones that join.
struct LogprobShared {
  Sums sums[LP_WARPS];
  float top_l[LP_WARPS];
  float bound[LP_WARPS];
  float v[LP_WARPS][32];
  int i[LP_WARPS][32];
};

template <typename T, bool TOP>
__global__ void __launch_bounds__(LP_WARPS * 32) k_logprob(const LogprobParams P) {
  __shared__ LogprobShared sh;
  extern __shared__ __align__(16) unsigned char lp_ring[];     // [warp][LP_STAGES] tiles
  cg::cluster_group cluster = cg::this_cluster();
  const int parts = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int64_t row = blockIdx.x / parts;
  const RowVectors<T> R((const T*)P.logits + row * P.ld, P.v);
  const int tiles = ceil_div(R.count(), 32 * Tile<T>::U), step = parts * warps;

  Sums a{-INFINITY, 0.f, 0.f};
  float top_l = -INFINITY;     // the largest l, NaNs aside
  TopList L;
  // Every warp of the CTA that has tiles has `share` values of at least its bound, so `top`
  // values of the row reach the least bound: none below it counts.
  const int busy = max(1, min(warps, tiles - rank * warps));
  const int share = TOP ? ceil_div(P.top, busy) : 1;
  volatile float* bound = sh.bound;
  if (TOP && warps > 1 && rank * warps + warp >= tiles) __syncthreads();     // the others' first tile
  uint4* ring = reinterpret_cast<uint4*>(lp_ring) + warp * LP_STAGES * 32 * Tile<T>::U;
  const int tile0 = rank * warps + warp;
  for (int n = 0; n < LP_STAGES - 1; ++n) {
    if (tile0 + n * step < tiles) Tile<T>::fetch(R, tile0 + n * step, lane, ring + n * 32 * Tile<T>::U);
    copies_group();
  }
  int stage = 0;
  for (int tile = tile0; tile < tiles; tile += step) {
    copies_left<LP_STAGES - 2>();
    __syncwarp();     // this tile is here for every lane, and the one before is done with
    {
      const int next = tile + (LP_STAGES - 1) * step, slot = stage == 0 ? LP_STAGES - 1 : stage - 1;
      if (next < tiles && next > tile) Tile<T>::fetch(R, next, lane, ring + slot * 32 * Tile<T>::U);
      copies_group();
    }
    const uint4* here = ring + stage * 32 * Tile<T>::U;
    stage = stage == LP_STAGES - 1 ? 0 : stage + 1;
    Tile<T> t;
    t.read(here, lane);
    const float tm = t.max();
    top_l = fmaxf(top_l, tm);
    if (tm >= NOTHING && tm <= USUAL) {
      const float m = ceilf(tm * LOG2E);
      if (m > a.m) a.to(m);
    }
    t.add(a);
    if constexpr (TOP) {
      const float real = tm == tm ? tm : -INFINITY;
      float least = -INFINITY;
      if (warps > 1) {
        if (tile == tile0) {     // the first: as many lanes' maxima to begin with
          const float b = nth_largest(real, share, lane);
          if (lane == 0) bound[warp] = b;
          __syncthreads();
        }
        least = bound[0];
        for (int w = 1; w < busy; ++w) least = fminf(least, bound[w]);
      }
      const bool full = L.at_i != INT_MAX;
      uint32_t lanes = __ballot_sync(0xffffffffu, (real > L.at_v || !full) && real >= least);
      if (lanes) {
        // `top` lanes have a value that reaches the top-th largest of their maxima
        if (__popc(lanes) >= P.top)
          least = fmaxf(least, nth_largest(real, P.top, lane));
        lanes = __ballot_sync(0xffffffffu, (lanes >> lane & 1u) && real >= least);
        while (lanes) {      // that lane's 32 elements, one a lane
          const int from = __ffs(lanes) - 1;
          lanes &= lanes - 1;
          constexpr int PER = Tile<T>::PER;
          const int at = (lane / PER * 32 + from) * PER + lane % PER;
          const float x = to_f32(reinterpret_cast<const T*>(here)[at]);
          // its index (below 0 before the row, at most 2^31 + 1023 as unsigned after it)
          const uint32_t e = (uint32_t)tile * LP_TILE + at - R.off;
          uint32_t c = __ballot_sync(0xffffffffu,
                                     e < (uint32_t)P.v && x >= least && before(x, (int)e, L.at_v, L.at_i));
          while (c) {
            const int src = __ffs(c) - 1;
            c &= c - 1;
            const float xv = __shfl_sync(0xffffffffu, x, src);
            const int xi = __shfl_sync(0xffffffffu, (int)e, src);
            if (before(xv, xi, L.at_v, L.at_i)) L.insert(xv, xi, lane, P.top);
          }
        }
        if (warps > 1 && lane == share - 1 && L.v > bound[warp]) bound[warp] = L.v;
      }
    }
  }
  a.join_warp();
#pragma unroll
  for (int o = 16; o; o >>= 1) top_l = fmaxf(top_l, __shfl_xor_sync(0xffffffffu, top_l, o));
  // Join: the warps of a CTA pairwise, then the cluster's CTAs by the first of them.
  auto leave = [&](int at) {
    if (lane == 0) {
      sh.sums[at] = a;
      sh.top_l[at] = top_l;
    }
    if (TOP) {
      sh.v[at][lane] = L.v;
      sh.i[at][lane] = L.i;
    }
  };
  for (int h = warps / 2; h; h /= 2) {
    if (warp >= h && warp < 2 * h) leave(warp);
    __syncthreads();
    if (warp < h) {
      a.join(sh.sums[warp + h]);
      top_l = fmaxf(top_l, sh.top_l[warp + h]);
      if (TOP) L.merge(sh.v[warp + h][lane], sh.i[warp + h][lane], lane);
    }
  }
  if (parts > 1) {
    if (warp == 0 && rank > 0) leave(0);
    cluster.sync();
    if (rank == 0 && warp == 0) {
      float v[7];
      int i[7];
#pragma unroll
      for (int p = 1; p < 8; ++p) {
        if (p >= parts) break;
        const LogprobShared* o = cluster.map_shared_rank(&sh, p);
        a.join(o->sums[0]);
        top_l = fmaxf(top_l, o->top_l[0]);
        if (TOP) {
          v[p - 1] = o->v[0][lane];
          i[p - 1] = o->i[0][lane];
        }
      }
#pragma unroll
      for (int p = 1; p < 8; ++p)
        if (TOP && p < parts) L.merge(v[p - 1], i[p - 1], lane);
    }
    cluster.sync();     // nobody's shared memory goes before it is read
  }
  if (rank > 0 || warp > 0) return;
  // log p = (l - base) - log s
  double base = (double)a.m * LN2;
  if (!(fabsf(top_l) <= USUAL)) {
    // A maximum that is too large, too low, or none at all: once more, by this warp.
    a = Sums{top_l, 0.f, 0.f};
    const float from = top_l == -INFINITY ? 0.f : top_l;     // then s is 0, or NaN
    for (int e = lane; e < P.v; e += 32) {
      const float d = max_nan((to_f32(R.row[e]) - from) * LOG2E, FAR), x = exp2_fast(d);
      a.s += x;
      a.u = fmaf(x, d, a.u);
    }
    a.s = warp_all(a.s, AddOp());
    a.u = warp_all(a.u, AddOp());
    base = (double)top_l;
  }
  const bool none = top_l == -INFINITY && a.s == 0.f;
  const float ls = logf(a.s);
  auto logp = [&](float l) { return none ? -INFINITY : (float)((double)l - base) - ls; };
  if (lane == 0) {
    P.lse[row] = none ? -INFINITY : (float)(base + (double)ls);
    P.entropy[row] = none ? 0.f : ls - a.u / a.s * (float)LN2;
    if (P.logp) {
      const int64_t at = P.targets[row];
      P.logp[row] = at < 0 || at >= P.v ? 0.f : logp(to_f32(R.row[at]));
    }
  }
  if (TOP && lane < P.top) {
    P.top_logp[row * P.top + lane] = logp(L.v);
    P.top_ids[row * P.top + lane] = L.i == INT_MAX ? -1 : L.i;
  }
}

template <typename T>
constexpr size_t lp_ring_bytes(int warps) { return (size_t)warps * LP_STAGES * LP_TILE * sizeof(T); }

template <typename T, bool TOP>
cudaError_t launch_logprob(const LogprobParams& P, cudaStream_t s) {
  static OncePerDevice once;
  const cudaError_t e = once([] {
    return cudaFuncSetAttribute(k_logprob<T, TOP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)lp_ring_bytes<T>(LP_WARPS));
  });
  if (e != cudaSuccess) return e;
  // Warps a row is shared by: as many as the GPU holds for all rows, at least four (their tiles
  // are in flight together; 4095 rows of 128256 bf16, top 20: 1 warp 241 us, 2: 218, 4: 214, 8: 238) and
  // no more than there are tiles.
  const int tiles = ceil_div(P.v, LP_TILE) + (P.v % 8 ? 1 : 0);
  const int want = std::min(tiles, std::max(4, ROW_SMS * 32 / P.rows));
  int warps = 1, parts = 1;
  while (warps < LP_WARPS && warps < want) warps *= 2;
  while (parts < 8 && parts * warps < want) parts *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)P.rows * parts);
  cfg.blockDim = dim3(32 * warps);
  cfg.dynamicSmemBytes = lp_ring_bytes<T>(warps);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = parts;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = parts > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, k_logprob<T, TOP>, P);
}

struct MaxOp {
  __device__ __forceinline__ float operator()(float a, float b) const { return max_nan(a, b); }
  static constexpr float none = -INFINITY;
};

struct LogprobBackParams {
  const void* logits;
  int64_t ld, ldd;
  const int64_t* targets;
  const float *lse, *entropy, *dlogp, *dentropy;
  void* d;
  int rows, v;
};

constexpr int LB_THREADS = 256;
constexpr int LB_ROWS_Y = 32768;  // rows along grid.y
constexpr int LB_VECTORS = 4;     // 16-byte vectors of logits per thread

// One read and one write of each element.
template <typename T>
__global__ void __launch_bounds__(LB_THREADS) k_logprob_back(const LogprobBackParams P) {
  __shared__ float slots[2][32];
  constexpr int PER = RowVectors<T>::PER;
  const int64_t row = blockIdx.y + (int64_t)blockIdx.z * LB_ROWS_Y;
  if (row >= P.rows) return;
  const RowVectors<T> R((const T*)P.logits + row * P.ld, P.v);
  T* d = (T*)P.d + row * P.ldd;
  const bool vec_out = (((uintptr_t)d ^ (uintptr_t)R.row) & 15) == 0;
  const int v0 = blockIdx.x * (LB_THREADS * LB_VECTORS) + threadIdx.x, count = R.count();
  uint4 r[LB_VECTORS];
#pragma unroll
  for (int u = 0; u < LB_VECTORS; ++u)
    if (R.inside(v0 + u * LB_THREADS)) r[u] = R.base[v0 + u * LB_THREADS];
  const float lse = P.lse[row];
  const int64_t at = P.targets ? P.targets[row] : -1;
  const float g = P.dlogp && at >= 0 && at < P.v ? P.dlogp[row] : 0.f;
  const float w = P.dentropy ? P.dentropy[row] : 0.f, H = P.dentropy ? P.entropy[row] : 0.f;
  const bool none = lse == -INFINITY;
  // log p = (l - m) - log s.  lse = m + log s in one number is enough unless it is so
  // large that its rounding is felt: such a row's m and s are formed again.
  // (By one CTA for the whole row, which may be overwritten: it reads all of it first.)
  float m = lse, ls = 0.f;
  const bool again = fabsf(lse) > LSE_EXACT && !none;
  if (again) {
    if (blockIdx.x > 0) return;
    m = -INFINITY;
    for (int e = threadIdx.x; e < P.v; e += LB_THREADS) m = max_nan(m, to_f32(R.row[e]));
    m = cta_all(m, MaxOp(), slots[0]);
    for (int e = threadIdx.x; e < P.v; e += LB_THREADS) ls += exp2_fast((to_f32(R.row[e]) - m) * LOG2E);
    ls = logf(cta_all(ls, AddOp(), slots[1]));
  }
  auto grad = [&](float l) {
    const float t = max_nan((l - m) - ls, FAR), p = exp2_fast(t * LOG2E);
    return none ? 0.f : -p * fmaf(w, t + H, g);
  };
  auto put = [&](int i, const uint4& q) {     // vector i of the row, q if it lies inside
    const int64_t e0 = R.first(i);
    if (R.inside(i)) {
      const uint32_t x[4] = {q.x, q.y, q.z, q.w};
      float o[PER];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (PER == 8) {
          o[2 * j] = grad(bf16_lo(x[j]));
          o[2 * j + 1] = grad(bf16_hi(x[j]));
        } else {
          o[j] = grad(__uint_as_float(x[j]));
        }
      }
      if (at >= e0 && at < e0 + PER) {
#pragma unroll
        for (int j = 0; j < PER; ++j)
          if (e0 + j == at && !none) o[j] += g;
      }
      if (vec_out) {
        if constexpr (PER == 8)
          store8(d + e0, o);
        else
          *reinterpret_cast<float4*>(d + e0) = make_float4(o[0], o[1], o[2], o[3]);
      } else {
#pragma unroll
        for (int j = 0; j < PER; ++j) d[e0 + j] = from_f32<T>(o[j]);
      }
    } else {
      for (int j = 0; j < PER; ++j) {
        const int64_t e = e0 + j;
        if (e < 0 || e >= P.v) continue;
        const float o = grad(to_f32(R.row[e]));
        d[e] = from_f32<T>(e == at && !none ? o + g : o);
      }
    }
  };
  if (again) {
    for (int i = threadIdx.x; i < count; i += LB_THREADS)
      put(i, R.inside(i) ? R.base[i] : make_uint4(0u, 0u, 0u, 0u));
    return;
  }
#pragma unroll
  for (int u = 0; u < LB_VECTORS; ++u) {
    const int i = v0 + u * LB_THREADS;
    if (i < count) put(i, r[u]);
  }
}

template <typename T>
void launch_logprob_back(const LogprobBackParams& P, cudaStream_t s) {
  const int64_t vectors = (P.v + (int64_t)RowVectors<T>::PER - 2) / RowVectors<T>::PER + 1;   // whatever the offset
  const dim3 grid((unsigned)((vectors + LB_THREADS * LB_VECTORS - 1) / (LB_THREADS * LB_VECTORS)),
                  (unsigned)std::min(P.rows, LB_ROWS_Y), (unsigned)ceil_div(P.rows, LB_ROWS_Y));
  k_logprob_back<T><<<grid, LB_THREADS, 0, s>>>(P);
}

}  // namespace
}  // namespace bakron

using namespace bakron;

extern "C" int bakron_token_logprobs(const void* logits, int dtype, int rows, int v, int64_t ldl,
                                     const int64_t* targets, int top, float* logp, float* entropy,
                                     float* lse, float* top_logp, int* top_ids, void* stream) {
  if ((dtype != BAKRON_F32 && dtype != BAKRON_BF16) || rows < 0 || v < 1 || v > V_MAX || top < 0 || top > TOP_MAX ||
      top > v || (targets != nullptr) != (logp != nullptr))
    return BAKRON_ERR_INVALID_ARG;
  if (rows == 0) return BAKRON_OK;
  if (!logits || ldl < v || !entropy || !lse || (top > 0 && (!top_logp || !top_ids)))
    return BAKRON_ERR_INVALID_ARG;
  LogprobParams P{logits, ldl, targets, rows, v, top, logp, entropy, lse, top_logp, top_ids};
  cudaStream_t s = (cudaStream_t)stream;
  const auto launch = dtype == BAKRON_F32 ? (top ? launch_logprob<float, true> : launch_logprob<float, false>)
                                          : (top ? launch_logprob<__nv_bfloat16, true>
                                                 : launch_logprob<__nv_bfloat16, false>);
  BK_CUDA_OK(launch(P, s));
  return BAKRON_OK;
}

extern "C" int bakron_token_logprobs_backward(const void* logits, int dtype, int rows, int v,
                                              int64_t ldl, const int64_t* targets, const float* lse,
                                              const float* dlogp, const float* entropy,
                                              const float* dentropy, void* dlogits, int64_t ldd,
                                              void* stream) {
  if ((dtype != BAKRON_F32 && dtype != BAKRON_BF16) || rows < 0 || v < 1 || v > V_MAX) return BAKRON_ERR_INVALID_ARG;
  if (rows == 0) return BAKRON_OK;
  if (!logits || !lse || !dlogits || ldl < v || ldd < v || (!dlogp && !dentropy) ||
      (dlogp && !targets) || (dentropy && !entropy))
    return BAKRON_ERR_INVALID_ARG;
  LogprobBackParams P{logits, ldl, ldd, targets, lse, entropy, dlogp, dentropy, dlogits, rows, v};
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == BAKRON_F32)
    launch_logprob_back<float>(P, s);
  else
    launch_logprob_back<__nv_bfloat16>(P, s);
  BK_CUDA_OK(cudaGetLastError());
  return BAKRON_OK;
}
