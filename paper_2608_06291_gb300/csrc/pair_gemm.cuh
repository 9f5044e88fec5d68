// A product of bf16 (or fp16) values on CTA pairs, C (M x N) = A B with fp32 sums, and what becomes of its
// tiles (the epilogue, a template parameter).  Used by the output head (head.cu) and by
// the gradient of the quantised product (linear_back.cu).
//
// A pair of CTAs computes 256 x bn tiles (bn <= 256) with M = 256 MMAs (cta_group::2): each
// CTA holds its own 128 rows of A and half of B's columns, so a 64-deep K block brings
// 16 + 16 KB into each SM's shared memory for 512 cycles of its tensor pipe; a lone CTA's
// 128 x 256 tile would need 16 + 32.  Warp 0 of each CTA loads (TMA, a ring of STAGES blocks), warp 1
// of the first CTA issues, eight warps of each take the finished sums out of TMEM, where two
// accumulators let the next sums' MMAs run meanwhile.  Pairs walk the tiles in a fixed order, so
// results do not depend on timing.
//
// In the tensor cores a sum is cut, not rounded, at each of its additions (one per 16 products), so a long one leans
// toward zero: of 2^20 products of one sign 0.65%, of 131072 7e-4.  It leaves TMEM after `group` K blocks and goes
// on in registers, where additions are rounded.
//
// Bound by the tensor pipe, busy in 93 to 95% of an SM's cycles while it works, at the clock that the power
// allows, and by the last round of tiles (87 to 92% of all cycles): 2048 x 32768 x 4096 284 to 296 us (1.86 to 1.94
// PFLOP/s), 4095 x 128256 x 4096 2.48 ms (1.73).
//
// Operands are K-major (a row's K values together) or MN-major (a K's rows together), read
// as they lie by TMA; what is out of range is filled with zeros.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cudaTypedefs.h>
#include <stdint.h>

#include "rowops.cuh"
#include "tc_gemm.cuh"
#include "tcgen05.cuh"

namespace bakron {

constexpr int PG_M = 256, PG_K = 64;            // rows of a tile, depth of a block
constexpr int PG_EPI_WARPS = 8;                 // per CTA: two per TMEM lane quarter
constexpr int PG_THREADS = 32 * (2 + PG_EPI_WARPS);
constexpr uint32_t PG_OPERAND = 16384;          // 128 rows of 64 bf16, or 64 rows of 2 x 64
constexpr uint32_t PG_STAGE = 2 * PG_OPERAND;
constexpr int PG_STAGES = 6;
constexpr uint32_t PG_OUT = 4096;               // an epilogue warp's 32 rows of 128 bytes
constexpr uint32_t PG_SMEM = PG_STAGES * PG_STAGE + PG_EPI_WARPS * PG_OUT + 1024 /*align*/ + 256 /*barriers*/;
static_assert(PG_SMEM <= 232448, "shared memory of an SM");

struct PairShape {
  int tm, tn;          // tiles
  int bn;              // columns of a tile: a multiple of 32, of 128 where B is MN-major
  int nk;              // K blocks in all
  int splits, per;     // ranges of K blocks, blocks of one (the last may be shorter)
  int group;           // K blocks summed in place in TMEM
  int band;            // row tiles walked side by side
  int half;            // operands are fp16
  int rows;            // rows of A: CTAs behind the last load none (K-major A)
  int a_rows;          // rows of a K-major A box (a multiple of 8, at most 128)
  int* status;         // gets the error of a wait that ran out; or, where there are
  int* flags;          // flags, each CTA's is written: the error or 0 (so nothing has to be cleared before)
  long long spin_cycles;
  __host__ __device__ int64_t items() const { return (int64_t)tm * tn * splits; }
};

// Item -> tile and range of K.
struct PairItem {
  int mt, nt, split, k0, n;
  __device__ __forceinline__ PairItem(const PairShape& S, int64_t item) {
    const int64_t tiles = (int64_t)S.tm * S.tn;
    split = (int)(item / tiles);
    const int64_t r = item % tiles;
    const int64_t in_band = (int64_t)S.band * S.tn;
    const int b = (int)(r / in_band);
    const int rem = (int)(r % in_band), bm = min(S.band, S.tm - b * S.band);
    nt = rem / bm;
    mt = b * S.band + rem % bm;
    k0 = split * S.per;
    n = min(S.per, S.nk - k0);
  }
};

// What an epilogue warp sees of a tile.
struct PairOut {
  int row;             // of C, this thread's (not below M in the last tiles: Epi checks)
  int row0;            // the warp's first row
  int nt, half;        // column tile, and which half of it
  int col, cols;       // first column and number of columns of this warp's half
  int split;
  unsigned char* stage;      // this warp's 4 KB
  int lane;
};

// Columns c..c+7 of this thread's row as 16 bytes of a staged box (128-byte rows, swizzled).
__device__ __forceinline__ uint4* staged(unsigned char* stage, int lane, int chunk) {
  return reinterpret_cast<uint4*>(stage + lane * 128 + ((chunk ^ (lane & 7)) << 4));
}
// The box may be written again (its last store has read it).
__device__ __forceinline__ void stage_free(int lane) {
  if (lane == 0) bulk_read_left<0>();
  __syncwarp();
}
// What the lanes wrote is visible to a TMA store.
__device__ __forceinline__ void stage_ready() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
}

// MN-major: 64-column (128-byte, swizzled) rows, one K each; 8-row groups 1024 bytes apart,
// the next 64 columns 8 KB on.
__device__ __forceinline__ uint64_t pair_desc(uint32_t addr, bool mn) {
  return mn ? (smem_desc(addr) & ~((uint64_t)0x3FFF << 16)) | ((uint64_t)(8192 >> 4) << 16) : smem_desc(addr);
}

template <class Epi, bool AMN, bool BMN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PG_THREADS, 1)
    k_pair_gemm(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
                const __grid_constant__ CUtensorMap mapO, const PairShape S, const typename Epi::Params E) {
  extern __shared__ __align__(1024) unsigned char pg_smem[];
  unsigned char* smem = (unsigned char*)(((uintptr_t)pg_smem + 1023) & ~(uintptr_t)1023);
  unsigned char* out = smem + PG_STAGES * PG_STAGE;
  uint64_t* bars = (uint64_t*)(out + PG_EPI_WARPS * PG_OUT);
  uint64_t* full = bars;                     // [STAGES] of the first CTA: both CTAs' halves are loaded
                                           // (its producer expects the bytes of both: an arrival from the
                                           // other CTA, a release at the cluster, cost 1000 cycles a block)
  uint64_t* empty = bars + PG_STAGES;        // [STAGES] read by its MMAs
  uint64_t* accF = bars + 2 * PG_STAGES;     // [2] sums finished
  uint64_t* accE = accF + 2;                 // [2] of the first CTA: sums read out by both
  uint64_t* done = accE + 2;                 // every MMA complete
  uint32_t* tmem_slot = (uint32_t*)(done + 1);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_rank();

  if (threadIdx.x == 0) {
    for (int s = 0; s < PG_STAGES; ++s) {
      mbar_init(&full[s], 1);      // the first CTA's producer, for both
      mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&accF[a], 1);
      mbar_init(&accE[a], 2 * PG_EPI_WARPS);
    }
    mbar_init(done, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  cluster_sync_all();      // both CTAs' barriers are there
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *tmem_slot;
  pdl_wait();         // so far nothing of the kernels before was touched
  const int64_t items = S.items(), step = gridDim.x >> 1, first = blockIdx.x >> 1;
  constexpr long long drain = 4000000000LL;      // about 2 s: the bound of the way out
  auto timed_out = [&]() {
    if (!S.flags) raise_status(S.status, BAKRON_ERR_TIMEOUT);
    *abort_flag = 1;
    st_peer_flag((const void*)abort_flag, rank);
  };
  auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {      // a warp; false: give up, here or elsewhere
    if (mbar_wait_warp(bar, parity, S.spin_cycles, abort_flag)) return true;
    if (lane == 0 && !*abort_flag) timed_out();
    __syncwarp();
    return false;
  };

  if (warp == 0) {
    // ------------------------------------------------------------ loads
    const uint32_t full0 = at_rank0(full);
    const uint32_t bbytes = (uint32_t)S.bn * 64u;      // bn / 2 columns of 64 bf16
    uint32_t s = 0, parity = 1;      // a fresh barrier's phase before the first counts as complete
    bool ok = true;
    for (int64_t item = first; item < items && ok; item += step) {
      const PairItem I(S, item);
      const int arow = I.mt * PG_M + rank * 128, bcol = I.nt * S.bn + rank * (S.bn >> 1);
      const bool load_a = AMN || arow < S.rows;
      // of both CTAs; the second one's first row is 128 on
      const uint32_t bytes = 2u * bbytes + (AMN ? 2u * PG_OPERAND
                                                : (uint32_t)S.a_rows * (arow + 128 < S.rows ? 256u : 128u));
      int k = I.k0 * PG_K;
      for (int i = 0; i < I.n; ++i, k += PG_K) {
        if (!wait(&empty[s], parity)) {
          ok = false;
          break;
        }
        if (elected()) {
          unsigned char *a = smem + s * PG_STAGE, *b = a + PG_OPERAND;
          const uint32_t bar = full0 + s * 8u;
          if (rank == 0) mbar_expect_tx(&full[s], bytes);
          if constexpr (AMN) {
            tma_load_2d_c2(a, &mapA, bar, arow, k);
            tma_load_2d_c2(a + 8192, &mapA, bar, arow + 64, k);
          } else {
            if (load_a) tma_load_2d_c2(a, &mapA, bar, k, arow);
          }
          if constexpr (BMN) {
            tma_load_2d_c2(b, &mapB, bar, bcol, k);
            if (S.bn > 128) tma_load_2d_c2(b + 8192, &mapB, bar, bcol + 64, k);
          } else {
            tma_load_2d_c2(b, &mapB, bar, k, bcol);
          }
        }
        __syncwarp();
        if (++s == PG_STAGES) s = 0, parity ^= 1u;
      }
    }
    if (*abort_flag) {      // copies in flight land within microseconds; wait about a millisecond
      const long long t0 = clock64();
      while (clock64() - t0 < 2000000LL) __nanosleep(1000);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs
    // The warp goes through the loop together and an elected lane issues: operands stay in uniform registers.
    if (rank == 0) {
      const uint32_t idesc = (S.half ? idesc_f16(PG_M, S.bn) : idesc_bf16(PG_M, S.bn)) | (AMN ? 1u << 15 : 0u) | (BMN ? 1u << 16 : 0u);
      const uint64_t da0 = pair_desc(smem_u32(smem), AMN), db0 = pair_desc(smem_u32(smem) + PG_OPERAND, BMN);
      constexpr uint64_t ka = AMN ? 2048 >> 4 : 2, kb = BMN ? 2048 >> 4 : 2;      // 16 K values on
      uint32_t s = 0, parity = 0, g = 0;
      bool ok = true;
      for (int64_t item = first; item < items && ok; item += step) {
        const PairItem I(S, item);
        int left = I.n;
        while (left > 0 && ok) {
          const int n = min(left, S.group);
          const uint32_t a = g & 1u, d = tmem + a * 256u;
          if (!wait(&accE[a], ((g >> 1) & 1u) ^ 1u)) {
            ok = false;
            break;
          }
          for (int i = 0; i < n; ++i) {
            if (!wait(&full[s], parity)) {
              ok = false;
              break;
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t da = da0 + (uint64_t)(s * (PG_STAGE >> 4)), db = db0 + (uint64_t)(s * (PG_STAGE >> 4));
            if (elected()) {
#pragma unroll
              for (int kk = 0; kk < 4; ++kk)
                mma_bf16_pair(d, da + kk * ka, db + kk * kb, idesc, (kk > 0 || i > 0) ? 1u : 0u);
              mma_commit_pair(&empty[s]);
              if (i == n - 1) mma_commit_pair(&accF[a]);
            }
            __syncwarp();
            if (++s == PG_STAGES) s = 0, parity ^= 1u;
          }
          left -= n;
          ++g;
        }
      }
      if (elected()) mma_commit_pair(done);
      __syncwarp();
    }
    if (lane == 0 && !mbar_wait_cluster(done, 0, drain)) timed_out();
    __syncwarp();
  } else {
    // ------------------------------------------------------------ epilogue
    const int q = warp & 3, half = (warp - 2) >> 2;
    const uint32_t accE0 = at_rank0(accE);
    PairOut O;
    O.lane = lane;
    O.half = half;
    O.stage = out + (warp - 2) * PG_OUT;
    O.cols = S.bn >> 1;
    uint32_t g = 0;
    bool ok = true;
    auto sums = [&](uint32_t a) -> bool {
      const bool r = wait(&accF[a], (g >> 1) & 1u);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      return r;
    };
    auto release = [&](uint32_t a) {
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) cmbar_arrive_tmem(accE0 + a * 8u);
    };
    for (int64_t item = first; item < items && ok; item += step) {
      const PairItem I(S, item);
      O.row0 = I.mt * PG_M + rank * 128 + q * 32;
      O.row = O.row0 + lane;
      O.nt = I.nt;
      O.split = I.split;
      O.col = I.nt * S.bn + half * O.cols;
      const uint32_t at = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * O.cols);
      float acc[128];
#pragma unroll
      for (int u = 0; u < 128; ++u) acc[u] = 0.f;
      const int ng = (I.n + S.group - 1) / S.group;
      for (int i = 0; i < ng; ++i, ++g) {
        const uint32_t a = g & 1u;
        if (!sums(a)) {
          ok = false;
          break;
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          if (c * 16 < O.cols) {
            uint32_t r[16];
            tmem_ld16(at + a * 256u + c * 16, r);
            tmem_wait_ld();
#pragma unroll
            for (int u = 0; u < 16; ++u) acc[16 * c + u] += __uint_as_float(r[u]);
          }
        }
        release(a);
      }
      if (ok && O.row0 < S.rows) Epi::tile(E, O, acc, &mapO);
    }
    if (lane == 0) bulk_commit_and_wait();
    __syncwarp();
  }
  pdl_trigger();      // (from the start, CTAs of the next kernel in the queue cost 77 tokens' forward pass 9 us of 46)
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  cluster_sync_all();      // neither CTA's memory or barriers go while the other may use them
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (threadIdx.x == 0 && S.flags) S.flags[blockIdx.x] = *abort_flag ? BAKRON_ERR_TIMEOUT : 0;
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// ------------------------------------------------------------------ epilogues
// fp32 sums to part [split][row][col], or added to what is there.
struct EpiF32 {
  struct Params {
    int add;
  };
  __device__ static __forceinline__ void tile(const Params& E, const PairOut& O, float (&acc)[128], const CUtensorMap* map) {
#pragma unroll
    for (int c = 0; c < 128; c += 32) {
      if (c >= O.cols) break;
      stage_free(O.lane);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float* v = acc + c + 4 * k;
        *reinterpret_cast<float4*>(staged(O.stage, O.lane, k)) = make_float4(v[0], v[1], v[2], v[3]);
      }
      stage_ready();
      if (O.lane == 0) {
        if (E.add)
          tma_reduce_add_3d(map, O.stage, O.col + c, O.row0, O.split);
        else
          tma_store_3d(map, O.stage, O.col + c, O.row0, O.split);
        bulk_commit();
      }
    }
  }
};

// 2^p, which may be beyond fp32, as two factors: v 2^p is v a b, exact but where the result is below 2^-126.
__device__ __forceinline__ float2 two_powers(int p) { return make_float2(scalbnf(1.f, p / 2), scalbnf(1.f, p - p / 2)); }
__device__ __forceinline__ float times(float v, float2 power) { return v * power.x * power.y; }

// bf16 results, to a TMA map or (where rows are not 16-byte aligned) element by element;
// with `first`, row r's sum gets the fp32 row first[r] of `more` added; with `power`, it is multiplied by power[r].
struct EpiBf16 {
  struct Params {
    __nv_bfloat16* c;      // null: TMA
    int64_t ldc;
    int rows, cols;
    const int* first;
    const float* more;
    int64_t ldmore;
    const float2* power;
  };
  __device__ static __forceinline__ void tile(const Params& E, const PairOut& O, float (&acc)[128], const CUtensorMap* map) {
    if (E.first && O.row < E.rows) {
      const int f = E.first[O.row];
      if (f != 0x7fffffff) {
        const float* more = E.more + f * E.ldmore;
#pragma unroll
        for (int u = 0; u < 128; ++u)
          if (u < O.cols && O.col + u < E.cols) acc[u] += more[O.col + u];
      }
    }
    if (E.power && O.row < E.rows) {
      const float2 power = E.power[O.row];
#pragma unroll
      for (int u = 0; u < 128; ++u) acc[u] = times(acc[u], power);
    }
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 128; c += 64) {
      if (c >= O.cols) break;
      stage_free(O.lane);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float* v = acc + c + 8 * k;
        *staged(O.stage, O.lane, k) =
            make_uint4(bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]), bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7]));
      }
      if (!E.c) {
        stage_ready();
        if (O.lane == 0) {
          tma_store_2d(map, O.stage, O.col + c, O.row0);
          bulk_commit();
        }
      } else {
        __syncwarp();
        for (int r = 0; r < 32 && O.row0 + r < E.rows; ++r)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int at = 32 * h + O.lane, col = O.col + c + at;
            const __nv_bfloat16 v = reinterpret_cast<const __nv_bfloat16*>(staged(O.stage, r, at >> 3))[at & 7];
            if (col < E.cols) E.c[(O.row0 + r) * E.ldc + col] = v;
          }
        __syncwarp();
      }
    }
  }
};

// ------------------------------------------------------------------ host side
// A row-major matrix of 16-bit values (or fp32: `planes` of them) in boxes of box_cols x box_rows.
inline bool pair_map(CUtensorMap* map, bool f32, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_cols,
                     int box_rows, int planes = 0) {
  if (!get_encode()) return false;
  const int es = f32 ? 4 : 2;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  const cuuint64_t strides[2] = {(cuuint64_t)(ld * es), (cuuint64_t)(ld * es) * (cuuint64_t)rows};
  const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1u}, ones[3] = {1u, 1u, 1u};
  return g_encode(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, planes ? 3 : 2,
                  const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Rows that TMA cannot read as they lie, copied to rows of whole 16 bytes.
static __global__ void __launch_bounds__(256) k_pair_copy(const __nv_bfloat16* from, int64_t ld, int64_t rows, int cols,
                                                          __nv_bfloat16* to, int64_t ldt) {
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x)
    for (int c = blockIdx.y * 256 + threadIdx.x; c < cols; c += 256 * gridDim.y) to[row * ldt + c] = from[row * ld + c];
}
inline cudaError_t pair_copy(const void* from, int64_t ld, int64_t rows, int cols, void* to, cudaStream_t s) {
  const dim3 grid((unsigned)(rows < 8 * ROW_SMS ? rows : 8 * ROW_SMS), (unsigned)(cols < 16 * 512 ? ceil_div(cols, 512) : 16));
  k_pair_copy<<<grid, 256, 0, s>>>((const __nv_bfloat16*)from, ld, rows, cols, (__nv_bfloat16*)to, round_up(cols, 8));
  return cudaGetLastError();
}

constexpr int PG_PAIRS = ROW_SMS / 2;
// K blocks summed in place where the result is rounded to bf16: 4096 products, cut by 256 additions.
constexpr int PG_GROUP = 64;

inline unsigned pair_ctas(const PairShape& S) {
  const int64_t items = S.items();
  return 2 * (unsigned)(items < PG_PAIRS ? items : PG_PAIRS);
}

template <class Epi, bool AMN, bool BMN>
cudaError_t pair_launch(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& o, const PairShape& S,
                        const typename Epi::Params& E, cudaStream_t s) {
  static OncePerDevice once;
  const cudaError_t e = once([] {
    return cudaFuncSetAttribute(k_pair_gemm<Epi, AMN, BMN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PG_SMEM);
  });
  if (e != cudaSuccess) return e;
  return launch_pdl(k_pair_gemm<Epi, AMN, BMN>, dim3(pair_ctas(S)), dim3(PG_THREADS), PG_SMEM, s, a, b, o, S, E);
}

}  // namespace bakron
