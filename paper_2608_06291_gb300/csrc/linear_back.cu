// bakron_linear_backward: dx = dy What, the gradient of y = x What^T at the tokens x,
// What_ij = s (c_ij - z) with the grid (s, z) of row i and j's group.
//
// The sum runs over What's rows, whose scales differ, so the scale cannot wait for the end of a
// sum as it does in the forward product: an operand is s (c - z), formed in fp32 and rounded
// once to bf16.
//
// Up to FUSED_TOKENS tokens: one kernel. D (128 columns of What x BN tokens) = A B with A the
// operands of a 128-column block, formed from the codes in shared memory as the MMAs take them
// (MN-major), and B the tokens' gradients, K-major by TMA.  What's rows are shared by the CTAs of a
// cluster, which add their parts through each other's shared memory, always in the same order.
// More tokens: the weight is written out in bf16 once, and read by the pair product.
#include <cooperative_groups.h>

#include <algorithm>

#include "linear.cuh"
#include "pair_gemm.cuh"

namespace cg = cooperative_groups;

namespace bakron {
namespace {

// ------------------------------------------------------------------ few tokens
constexpr int FB_WARPS = 8;                      // expand, then write out
constexpr int FB_THREADS = 32 * (2 + FB_WARPS);  // warp 0 loads gradients, warp 1 issues MMAs
constexpr int FB_K = 64;                         // rows of What of a stage
constexpr uint32_t FB_A = FB_K * 128 * 2;        // its operands: 2 x 64 columns, [row][64]
constexpr int FB_STAGES = 4;

struct FusedParams {
  const unsigned char* codes;
  const float* scales;
  const uint8_t* zeros;
  int64_t mp;
  int kblocks, chunks, G;
  int rows, n, bn;         // tokens, columns, tokens of a tile (a multiple of 16)
  int nk, per;             // stages in all, of a CTA of the cluster
  __nv_bfloat16* dx;
  int64_t ldx;
  int vec;                 // dx can be written 16 bytes at a time
  int* status;
  long long spin_cycles;
};

// Two values c - z times s, rounded once: s = hi + lo, and what the small product loses is
// far below the sum's rounding.
__device__ __forceinline__ uint32_t scaled(uint32_t v, __nv_bfloat162 hi, __nv_bfloat162 lo) {
  const __nv_bfloat162 c = *reinterpret_cast<__nv_bfloat162*>(&v);
  const __nv_bfloat162 r = __hfma2(c, hi, __hmul2(c, lo));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Two 8-bit codes of a pair as c - z in fp16 (1024 + c is exact there), times s in fp32.
__device__ __forceinline__ uint32_t scaled8(uint32_t w, int odd, __half2 z1024, float s) {
  uint32_t u = __byte_perm(w, 0x64646464u, odd ? 0x4341 : 0x4240);
  const float2 c = __half22float2(__hsub2(*reinterpret_cast<__half2*>(&u), z1024));
  return bf16_pack(c.x * s, c.y * s);
}

// What a thread needs of a stage: a row's unit (two with 8 bits a code), its grids.
template <bool W8, bool ONE>
struct Piece {
  uint4 u[W8 ? 2 : 1];
  float s[ONE ? 1 : 4];
  uint8_t z[ONE ? 1 : 4];
};

// ONE: the 128 columns of a block have one grid a row.
template <bool W8, bool ONE>
__global__ void __launch_bounds__(FB_THREADS, 2) k_back_fused(const __grid_constant__ CUtensorMap map, const FusedParams P) {
  extern __shared__ __align__(1024) unsigned char fb_smem[];
  unsigned char* smem = (unsigned char*)(((uintptr_t)fb_smem + 1023) & ~(uintptr_t)1023);
  const uint32_t stage_bytes = FB_A + (uint32_t)P.bn * 128u;
  __shared__ uint64_t full[FB_STAGES], formed[FB_STAGES], empty[FB_STAGES], done;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  cg::cluster_group cluster = cg::this_cluster();
  const int splits = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
  const int cb = blockIdx.x / splits, tok0 = blockIdx.y * P.bn;
  const int k0 = part * P.per, nk = max(0, min(P.per, P.nk - k0));
  const uint32_t cols = P.bn <= 32 ? 32u : P.bn <= 64 ? 64u : P.bn <= 128 ? 128u : 256u;

  if (threadIdx.x == 0) {
    for (int i = 0; i < FB_STAGES; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&formed[i], FB_WARPS);
      mbar_init(&empty[i], 1);
    }
    mbar_init(&done, 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  constexpr long long drain = 4000000000LL;      // about 2 s: the bound of the way out
  auto timed_out = [&]() {
    pdl_wait();      // the status is cleared by the kernel before
    raise_status(P.status, BAKRON_ERR_TIMEOUT);
    abort_flag = 1;
  };
  // a warp's wait; `out`: on the way out, whatever happened elsewhere
  auto wait = [&](uint64_t* bar, uint32_t parity, bool out = false) -> bool {
    if (mbar_wait_warp(bar, parity, out ? drain : P.spin_cycles, out ? nullptr : &abort_flag)) return true;
    if (lane == 0 && !abort_flag) timed_out();
    __syncwarp();
    return false;
  };

  if (warp == 0) {
    // ------------------------------------------------------------ gradients
    int it = 0;
    for (; it < nk; ++it) {
      const int s = it % FB_STAGES;
      if (it >= FB_STAGES && !wait(&empty[s], (uint32_t)(it / FB_STAGES - 1) & 1u)) break;
      if (elected()) {
        mbar_expect_tx(&full[s], (uint32_t)P.bn * 128u);
        tma_load_2d(smem + s * stage_bytes + FB_A, &map, &full[s], (k0 + it) * FB_K, tok0);
      }
      __syncwarp();
    }
    // every copy has landed before the CTA (and its shared memory) goes
    for (int j = max(0, it - FB_STAGES); j < it; ++j) wait(&full[j % FB_STAGES], (uint32_t)(j / FB_STAGES) & 1u, true);
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs
    const uint32_t idesc = idesc_bf16(128, P.bn) | 1u << 15;
    for (int it = 0; it < nk; ++it) {
      const int s = it % FB_STAGES;
      const uint32_t parity = (uint32_t)(it / FB_STAGES) & 1u;
      if (!wait(&full[s], parity) || !wait(&formed[s], parity)) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t at = smem_u32(smem) + s * stage_bytes;
      const uint64_t a = pair_desc(at, true), b = smem_desc(at + FB_A);
      if (elected()) {
#pragma unroll
        for (int k = 0; k < 4; ++k) mma_bf16(tmem, a + k * (2048 >> 4), b + k * 2, idesc, it > 0 || k > 0 ? 1u : 0u);
        mma_commit(&empty[s]);
      }
      __syncwarp();
    }
    if (elected()) mma_commit(&done);
    __syncwarp();
    wait(&done, 0, true);
  } else {
    // ------------------------------------------------------------ operands
    // A thread takes a row's 32 codes of a stage: lanes 0-7 eight rows of unit 0, the next eight
    // the same rows of unit 1, ..., so that loads are whole lines and the 16-byte stores of
    // eight lanes cover the banks.
    constexpr int UNITS = W8 ? 8 : 4, D = W8 || !ONE ? 2 : 4;      // stages ahead: as registers allow
    const int t = lane >> 3, r0 = (warp - 2) * 8 + (lane & 7);
    int grid[ONE ? 1 : 4];
#pragma unroll
    for (int j = 0; j < (ONE ? 1 : 4); ++j) grid[j] = P.G == 1 ? 0 : min((cb * 4 + j) / P.chunks, P.G - 1);
    auto load = [&](int it, Piece<W8, ONE>& to) {
      const int64_t row = (int64_t)(k0 + it) * FB_K + r0;
      const uint4* at = reinterpret_cast<const uint4*>(P.codes) +
                        (((row >> 7) * P.kblocks + cb) * UNITS + t) * LIN_BLOCK + (row & 127);
#pragma unroll
      for (int h = 0; h < (W8 ? 2 : 1); ++h) to.u[h] = __ldg(at + h * 4 * LIN_BLOCK);
#pragma unroll
      for (int j = 0; j < (ONE ? 1 : 4); ++j) {
        to.s[j] = __ldg(P.scales + grid[j] * P.mp + row);
        to.z[j] = __ldg(P.zeros + grid[j] * P.mp + row);
      }
    };
    Piece<W8, ONE> next[D];
#pragma unroll
    for (int q = 0; q < D; ++q)
      if (q < nk) load(q, next[q]);
    bool ok = true;
    for (int base = 0; base < nk && ok; base += FB_STAGES) {
#pragma unroll
      for (int q = 0; q < FB_STAGES; ++q) {
        const int it = base + q;
        if (it >= nk || !ok) break;
        const Piece<W8, ONE> here = next[q % D];
        if (it + D < nk) load(it + D, next[q % D]);
        if (base > 0 && !wait(&empty[q], (uint32_t)(base / FB_STAGES - 1) & 1u)) {
          ok = false;
          break;
        }
        unsigned char* a = smem + q * stage_bytes + r0 * 128;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float sf = here.s[ONE ? 0 : j], zf = (float)here.z[ONE ? 0 : j];
          uint32_t o[4];
          if constexpr (W8) {
            const __half2 z = __float2half2_rn(1024.f + zf);
            const uint32_t* w = reinterpret_cast<const uint32_t*>(&here.u[j >> 1]);
#pragma unroll
            for (int p = 0; p < 4; ++p) o[p] = scaled8(w[2 * (j & 1) + (p >> 1)], p & 1, z, sf);
          } else {
            const __nv_bfloat162 z = __float2bfloat162_rn(128.f + zf), hi = __float2bfloat162_rn(sf);
            const __nv_bfloat162 lo = __float2bfloat162_rn(sf - __low2float(hi));
            const uint32_t w = reinterpret_cast<const uint32_t*>(&here.u[0])[j];
#pragma unroll
            for (int p = 0; p < 4; ++p) o[p] = scaled(pair4(w, p, z), hi, lo);
          }
          *reinterpret_cast<uint4*>(a + (j >> 1) * 8192 + (((4 * (j & 1) + t) ^ (r0 & 7)) << 4)) =
              make_uint4(o[0], o[1], o[2], o[3]);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(&formed[q]);
      }
    }
    if (ok) wait(&done, 0);
  }
  // ------------------------------------------------------------ sums
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();      // the stages are free: the CTA's sums take their place, [token][128 columns]
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  float* mine = reinterpret_cast<float*>(smem);
  if (warp >= 2) {
    const int q = warp & 3, half = (warp - 2) >> 2, each = P.bn >> 1;
    if (nk > 0) {
      for (int c = half * each; c < (half + 1) * each; c += 8) {
        uint32_t r[8];
        tmem_ld8(tmem + ((uint32_t)(q * 32) << 16) + c, r);
        tmem_wait_ld();
#pragma unroll
        for (int u = 0; u < 8; ++u) mine[(c + u) * 128 + q * 32 + lane] = __uint_as_float(r[u]);
      }
    } else {
      for (int c = half * each; c < (half + 1) * each; ++c) mine[c * 128 + q * 32 + lane] = 0.f;
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  if (splits > 1)
    cluster.sync();
  else
    __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
  const int tokens = min(P.bn, P.rows - tok0);
  for (int i = part * FB_THREADS + (int)threadIdx.x; i < tokens * 16; i += splits * FB_THREADS) {
    const int tok = i >> 4, c = (i & 15) * 8;
    float v[8] = {};
    for (int p = 0; p < splits; ++p) {
      float u[8];
      load8((splits > 1 ? cluster.map_shared_rank(mine, p) : mine) + tok * 128 + c, u);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += u[k];
    }
    const int col = cb * 128 + c;
    __nv_bfloat16* out = P.dx + (int64_t)(tok0 + tok) * P.ldx + col;
    if (P.vec && col + 8 <= P.n) {
      store8(out, v);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (col + k < P.n) out[k] = __float2bfloat16_rn(v[k]);
    }
  }
  if (splits > 1) cluster.sync();      // nobody's shared memory goes before it is read
}

// ------------------------------------------------------------------ many tokens

struct ExpandParams {
  const unsigned char* codes;
  const float* scales;
  const uint8_t* zeros;
  int m, kblocks, chunks, G;
  int64_t mp;
  __nv_bfloat16* w;
  int64_t ldw;      // a multiple of 128
};

// What in bf16, row by row.  A thread takes a 16-byte unit; four lanes have a row's chunk together.
template <bool W8>
__global__ void __launch_bounds__(256) k_expand(const ExpandParams P) {
  constexpr int UNITS = W8 ? 8 : 4;
  const int t = threadIdx.x & 3;
  const int64_t i = blockIdx.x * 64 + (threadIdx.x >> 2);      // [row block][column block][half][row in the block]
  const int in = (int)(i % LIN_BLOCK);
  const int64_t rest = i / LIN_BLOCK;
  const int half = (int)(rest % (UNITS / 4)), kb = (int)(rest / (UNITS / 4) % P.kblocks);
  const int64_t rb = rest / (UNITS / 4) / P.kblocks, row = rb * LIN_BLOCK + in;
  if (row >= P.m) return;
  const uint4 u = reinterpret_cast<const uint4*>(P.codes)[((rb * P.kblocks + kb) * UNITS + half * 4 + t) * LIN_BLOCK + in];
  const uint32_t words[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int j = 0; j < (W8 ? 2 : 4); ++j) {
    const int chunk = kb * 4 + (W8 ? half * 2 : 0) + j, grid = P.G == 1 ? 0 : min(chunk / P.chunks, P.G - 1);
    const float s = P.scales[grid * P.mp + row], z = (float)P.zeros[grid * P.mp + row];
    const __nv_bfloat162 zz = __float2bfloat162_rn(z + (W8 ? 0.f : 128.f));
    uint32_t o[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint32_t c = W8 ? pair8(words[2 * j], words[2 * j + 1], p, zz) : pair4(words[j], p, zz);
      o[p] = bf16_pack(bf16_lo(c) * s, bf16_hi(c) * s);
    }
    *reinterpret_cast<uint4*>(P.w + row * P.ldw + chunk * 32 + 8 * t) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

__global__ void __launch_bounds__(256) k_back_copy(const __nv_bfloat16* from, int64_t ld, int rows, int m, __nv_bfloat16* to,
                                                   int64_t ldt) {
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x)
    for (int c = threadIdx.x; c < m; c += blockDim.x) to[row * ldt + c] = from[row * ld + c];
}

constexpr int FUSED_TOKENS = 512;

struct BackLayout {
  size_t dy = 0, w, bytes;
  bool copy;
  int64_t ldw;
  BackLayout(const void* p, int rows, int64_t ld, int m, int n) {
    size_t at = 256;
    copy = !aligned16(p, rows > 1 ? ld * 2 : 0);
    if (copy) {
      dy = at;
      at += align256((size_t)rows * round_up(m, 8) * 2);
    }
    w = at;
    ldw = round_up(n, LIN_BLOCK);
    bytes = rows > FUSED_TOKENS ? w + align256((size_t)m * ldw * 2) : at;
  }
};

constexpr uint32_t FB_SMEM_MAX = FB_STAGES * (FB_A + 256 * 128) + 1024;

// Tokens of a tile: as even as tiles of at most 256 allow.
int fused_bn(int rows) { return (int)round_up(ceil_div(rows, ceil_div(rows, 256)), 16); }
// CTAs of a cluster: What's rows are split until two CTAs an SM are busy (one, where tiles are tall).
int fused_splits(int rows, int m, int n) {
  const int bn = fused_bn(rows), tiles = ceil_div(n, 128) * ceil_div(rows, bn);
  const int slots = ROW_SMS * (2 * (FB_STAGES * (FB_A + bn * 128) + 2048) <= 227 * 1024 ? 2 : 1);
  return std::max(1, std::min({slots / tiles, ceil_div(m, 2 * FB_K), 8}));
}

template <bool W8, bool ONE>
cudaError_t fused_launch(const CUtensorMap& map, const FusedParams& P, int splits, cudaStream_t s) {
  static OncePerDevice once;
  const cudaError_t e = once([] {
    return cudaFuncSetAttribute(k_back_fused<W8, ONE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)FB_SMEM_MAX);
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(ceil_div(P.n, 128) * splits), (unsigned)ceil_div(P.rows, P.bn));
  cfg.blockDim = dim3(FB_THREADS);
  // the stages, or the sums that take their place
  cfg.dynamicSmemBytes = std::max<size_t>(FB_STAGES * (FB_A + (size_t)P.bn * 128), (size_t)P.bn * 512) + 1024;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, k_back_fused<W8, ONE>, map, P);
}

constexpr int LB_MAX_DIM = 1 << 17, LB_MAX_ROWS = 1 << 24;

bool back_ok(int rows, int m, int n, int qmax, int group_size) {
  return rows >= 0 && rows <= LB_MAX_ROWS && m >= 1 && n >= 1 && m <= LB_MAX_DIM && n <= LB_MAX_DIM && qmax >= 1 &&
         qmax <= 255 && (group_size == 0 || (group_size > 0 && group_size % 32 == 0 && n % group_size == 0));
}

}  // namespace
}  // namespace bakron

using namespace bakron;

extern "C" size_t bakron_linear_backward_workspace_bytes(const void* dy, int rows, int64_t lddy, int m, int n, int qmax,
                                                         int group_size) {
  return back_ok(rows, m, n, qmax, group_size) && rows > 0 ? BackLayout(dy, rows, lddy, m, n).bytes : 0;
}

extern "C" int bakron_linear_backward(const void* dy, int rows, int64_t lddy, const void* packed, int m, int n, int qmax,
                                      int group_size, void* dx, int64_t lddx, void* workspace, size_t workspace_bytes,
                                      int sync, void* stream) {
  if (!back_ok(rows, m, n, qmax, group_size)) return BAKRON_ERR_INVALID_ARG;
  if (rows == 0) return BAKRON_OK;
  if (!dy || !packed || !dx || lddy < m || lddx < n || (uintptr_t)packed % 16 != 0 || (uintptr_t)dy % 2 != 0 ||
      (uintptr_t)dx % 2 != 0 || !workspace || (uintptr_t)workspace % 16 != 0)
    return BAKRON_ERR_INVALID_ARG;
  const BackLayout B(dy, rows, lddy, m, n);
  if (workspace_bytes < B.bytes) return BAKRON_ERR_WORKSPACE;
  const WeightLayout L(m, n, qmax, group_size);
  const unsigned char* p = (const unsigned char*)packed;
  cudaStream_t s = (cudaStream_t)stream;
  char* ws = (char*)workspace;
  if (B.copy) {
    k_back_copy<<<(unsigned)std::min(rows, 8 * ROW_SMS), 256, 0, s>>>((const __nv_bfloat16*)dy, lddy, rows, m,
                                                                      (__nv_bfloat16*)(ws + B.dy), round_up(m, 8));
    BK_CUDA_OK(cudaGetLastError());
    dy = ws + B.dy;
    lddy = round_up(m, 8);
  }
  k_clear_status<<<1, 1, 0, s>>>((int*)ws);
  BK_CUDA_OK(cudaGetLastError());
  const int64_t ldmap = rows > 1 ? lddy : round_up(m, 8);
  CUtensorMap a, b, o;
  if (rows <= FUSED_TOKENS) {
    FusedParams F{p + L.off_codes, (const float*)(p + L.off_scales), p + L.off_zeros, L.mp, (int)(L.np / LIN_BLOCK),
                  L.G == 1 ? (int)(L.np / 32) : L.group / 32, (int)L.G, rows, n, fused_bn(rows), ceil_div(m, FB_K), 0,
                  (__nv_bfloat16*)dx, lddx, aligned16(dx, rows > 1 ? lddx * 2 : 0), (int*)ws, spin_cycles_from_env()};
    const int splits = fused_splits(rows, m, n);
    F.per = ceil_div(F.nk, splits);
    if (!pair_map(&a, false, dy, rows, m, ldmap, FB_K, F.bn)) return BAKRON_ERR_CUDA;
    const bool one = L.G == 1 || L.group % LIN_BLOCK == 0;
    BK_CUDA_OK(L.bytes8 ? (one ? fused_launch<true, true>(a, F, splits, s) : fused_launch<true, false>(a, F, splits, s))
                        : (one ? fused_launch<false, true>(a, F, splits, s) : fused_launch<false, false>(a, F, splits, s)));
    return sync ? bakron_read_status(workspace, stream) : BAKRON_OK;
  }
  ExpandParams E{p + L.off_codes, (const float*)(p + L.off_scales), p + L.off_zeros, m, (int)(L.np / LIN_BLOCK),
                 L.G == 1 ? (int)(L.np / 32) : L.group / 32, (int)L.G, L.mp, (__nv_bfloat16*)(ws + B.w), B.ldw};
  const unsigned ctas = (unsigned)(L.mp * E.kblocks * (L.units / 4) / 64);
  L.bytes8 ? k_expand<true><<<ctas, 256, 0, s>>>(E) : k_expand<false><<<ctas, 256, 0, s>>>(E);
  BK_CUDA_OK(cudaGetLastError());
  PairShape S{};
  S.tm = ceil_div(rows, PG_M);
  S.tn = ceil_div(n, 256);
  S.bn = 256;
  S.nk = S.per = S.group = ceil_div(m, PG_K);
  S.splits = 1;
  S.band = 16;
  S.rows = rows;
  S.a_rows = rows >= 128 ? 128 : (int)round_up(rows, 8);
  S.status = (int*)ws;
  S.spin_cycles = spin_cycles_from_env();
  const bool tma = aligned16(dx, rows > 1 ? lddx * 2 : 0);
  if (!pair_map(&a, false, dy, rows, m, ldmap, PG_K, S.a_rows) ||
      !pair_map(&b, false, E.w, m, n, B.ldw, 64, PG_K) ||
      (tma && !pair_map(&o, false, dx, rows, n, rows > 1 ? lddx : round_up(n, 8), 64, 32)))
    return BAKRON_ERR_CUDA;
  EpiBf16::Params T{tma ? nullptr : (__nv_bfloat16*)dx, lddx, rows, n, nullptr, nullptr, 0};
  BK_CUDA_OK((pair_launch<EpiBf16, false, true>(a, b, tma ? o : a, S, T, s)));
  return sync ? bakron_read_status(workspace, stream) : BAKRON_OK;
}
