// bakron_linear for many tokens: What's codes become exact operands of the tensor cores.
//
// D (128 rows of What x BN tokens) += A B: A, the integers c - z, is written into TMEM by
// four expanding warps (a thread is a row: its zero is a register), B, the tokens, lies
// in shared memory as TMA leaves it (K-major, 128-byte swizzle).  So a code is read once
// as 4 or 8 bits and never goes through shared memory in its expanded form.
//   bf16 tokens: kind::f16, c - z in bf16 (|c - z| <= 255: exact).
//   e4m3 tokens: kind::f8f6f4, c - z in e4m3 (|c - z| <= 15: exact).  e4m3 is linear up to
//     16 2^-9 (byte i is i 2^-9), so c - z is a sign and |c - z| itself, four codes at a time.
//     (The odd integer 2 c - 15, with 7.5 - z times the sum of a token's values, is cheaper to
//     form, 830 us for 845 at 4096 x 28672 x 8192 with GELU, but its two parts cancel: a row with
//     few codes beside its zero loses most of its bits.  In groups of 128, without GELU, it took
//     2.19 ms, this 1.60.)
// A grid's sum (a segment; 64 MMAs' columns where a row has one grid) accumulates in TMEM
// from zero; the epilogue warps multiply it by the grid's scale and add it in fp32
// registers while the next one is formed.
//
// Roles: warp 0 loads tokens, warp 2 codes, warp 3 what a grid needs, warp 1 issues the MMAs, warps 4-7 and 8-11
// expand (half of a stage each), warps 12-19 (two per lane quarter of TMEM) sum and write out.  CTAs are persistent, or, where there are fewer tiles than SMs, up to 8 CTAs of a
// cluster share a tile's columns and add their parts through each other's shared memory,
// always in the same order.
#include <cooperative_groups.h>
#include <cuda.h>

#include <algorithm>

#include "linear.cuh"
#include "tc_gemm.cuh"
#include "tcgen05.cuh"

namespace cg = cooperative_groups;

namespace bakron {
namespace {

constexpr int SEG_MMAS = 64;             // MMAs of a segment where a row has one grid: 1024 (2048) columns
constexpr int TOKEN_GROUP = 16;          // token tiles that share a pass over the weight

// The way out: an epilogue warp's 32 rows of 8 tokens at a time, token by token.
constexpr int STAGE_LD = 36;             // floats of a token: 16-byte reads of 8 lanes meet no bank twice

// A stage is 256 bytes of a token (two boxes of 128): 128 bf16 columns or 256 e4m3 columns,
// eight MMAs.  What an iteration of the issuing warp costs beside its MMAs (barriers,
// fence, commit: some 200 cycles) is only partly hidden by the MMAs in the queue, so
// a stage has as many as TMEM has room for (four a stage: 4096 x 28672 x 8192 in bf16 1.67 ms).
template <int BN_, bool W8_, bool X8_>
struct TcShape {
  static constexpr int BN = BN_;
  static constexpr bool W8 = W8_, X8 = X8_;
  static constexpr int EW = 2;                           // warpgroups that sum
  static constexpr int THREADS = 128 * (3 + EW);
  static constexpr int LAUNCH_REGS = 96;                 // of a thread: 65536 / THREADS, in steps of 8
  static constexpr int NACC = 2;                         // accumulators of BN columns
  static constexpr int NA = BN > 128 ? 2 : 4;            // A stages, 64 TMEM columns each
  static constexpr int ACC_COLS = NACC * BN;
  static constexpr int BPS = X8 ? 2 : 1;                 // 128-column blocks of a stage
  static constexpr int MPC = X8 ? 1 : 2;                 // MMAs of a 32-column chunk
  static constexpr uint32_t BOX = BN * 128;              // bytes of a box of tokens
  static constexpr uint32_t WS = W8 ? 16384 : 8192;      // bytes of a block's codes
  static constexpr int NX = BN > 128 ? 3 : 4;
  static constexpr int NW = W8 ? (BN > 128 ? 3 : BN > 64 ? 4 : 6) : BN > 128 ? 7 : BN > 64 ? 8 : 12;
  static constexpr int COLS = BN / EW;                   // columns an epilogue warp sums
  static constexpr uint32_t STAGE_BYTES = 4 * EW * 8 * STAGE_LD * 4;
  static constexpr uint32_t GS = LIN_BLOCK * 4;          // what the epilogue needs of a grid: the rows' scales
  static constexpr int NG = BN > 128 ? 8 : 16;           // enough for a load's way from memory
  static constexpr int ND = 4;                           // barriers of "the stage's MMAs are done"
  // behind the rings: the barriers, then TMEM's address and the abort flag
  static constexpr int BARRIERS = NX + ND + 2 * NW + NA + 2 * NACC + 2 * NG + 1;
  static constexpr uint32_t RINGS = 2 * NX * BOX + NW * WS + STAGE_BYTES + NG * GS;
  static constexpr uint32_t SMEM_USED = 1024 /*align*/ + RINGS + BARRIERS * 8 + 8;
  static constexpr uint32_t SMEM = SMEM_USED < 120 * 1024 ? 120 * 1024 : SMEM_USED;   // one CTA an SM
  // registers a thread of each warpgroup, out of those launched with
  static constexpr bool SPLIT_REGS = BN >= 128;
  static constexpr int R_LOAD = 56, R_EXPAND = 64, R_SUM = 144;
  static_assert((ND & (ND - 1)) == 0 && (NACC & (NACC - 1)) == 0, "masks");
  static_assert(ND >= NX && ND >= NA, "a barrier's phase is waited for before the next one can end");
  static_assert(ACC_COLS + NA * 64 <= 512, "TMEM");
  static_assert(SMEM <= 232448, "shared memory");
  static_assert(RINGS % 8 == 0 && (NW * WS) % 16 == 0 && GS % 16 == 0, "barriers and bulk copies are aligned");
  static_assert(R_LOAD + 2 * R_EXPAND + EW * R_SUM <= (3 + EW) * LAUNCH_REGS, "registers");
  static_assert((uint32_t)BN * 128 * 4 <= 2 * NX * BOX || BN > 128, "parts of a split tile");
};

struct TcParams {
  LinearParams L;
  int row_tiles, token_tiles, splits, per;   // per: 128-column blocks of a split's part
  uint32_t by_chunks;     // 2^32 / (chunks of a grid), rounded up: chunk / chunks by a product; 0 for 1
  int seg_chunks, segs;   // chunks of a segment; how many there are (the last takes the rest)
  long long spin_cycles;
};

// Whether a phase is over, without waiting (mbar_test's try_wait may hold the thread a while).
__device__ __forceinline__ bool mbar_look(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}

// A warp's wait for two barriers, every lane testing (the vote keeps the control flow
// uniform); gives up after `limit` cycles, or once another role has.
__device__ __forceinline__ bool tc_wait(uint64_t* bar, uint32_t parity, uint64_t* bar2, uint32_t parity2, long long limit,
                                        volatile int* abort_flag) {
  const bool now = mbar_look(bar, parity) && (bar2 == bar || mbar_look(bar2, parity2));
  if (__all_sync(0xffffffffu, now)) return true;
  const long long t0 = clock64();
  while (true) {
    if (__any_sync(0xffffffffu, *abort_flag || clock64() - t0 > limit)) return false;
    const bool a = mbar_test(bar, parity), b = bar2 == bar || mbar_test(bar2, parity2);
    if (__all_sync(0xffffffffu, a && b)) return true;
  }
}

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
          smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
      : "memory");
}

// 16 columns of this thread's TMEM lane.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}

// 16 columns of this thread's TMEM lane; valid after tmem_wait_ld().
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}

// D += A B, A in TMEM: 16 bf16 or 32 e4m3 columns, 8 TMEM columns either way.
template <bool X8>
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  if constexpr (X8)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// One lane of a whole warp, the way the compiler knows it: what it does keeps its operands
// in uniform registers.
__device__ __forceinline__ bool elected() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e != 0;
}

// kind::f8f6f4: D fp32, A and B e4m3 (format 0), K-major, 128 x N.
__host__ __device__ constexpr uint32_t idesc_e4m3(int N) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

template <int R>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R)); }
template <int R>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R)); }

// The segment of the chunks as they go by.
struct Segments {
  int seg, left, each, last;
  __device__ Segments(const TcParams& P, int chunk) : each(P.seg_chunks), last(P.segs - 1) {
    seg = min(chunk / each, last);
    left = seg == last ? INT_MAX : (seg + 1) * each - chunk;
  }
  __device__ __forceinline__ void next() {
    ++seg;
    left = seg == last ? INT_MAX : each;
  }
};

// The 8 codes of a word as e4m3 (c - z) 2^-9, in the columns' order; z in every byte of zz.
// The comparison as a product keeps it off the integer pipe (an addition there: 907 us for 845).
__device__ __forceinline__ void minus_zero8(uint32_t w, uint32_t zz, uint32_t& o0, uint32_t& o1) {
  auto four = [zz](uint32_t u) {      // columns 0 4 1 5, or 2 6 3 7
    const uint32_t c = u & 0x0F0F0F0Fu, t = c * 7u + (0x80808080u - 7u * zz);   // bit 7 of a byte: c >= z
    return __vabsdiffu4(c, zz) | (~t & 0x80808080u);
  };
  const uint32_t a = four(w), b = four(w >> 4);
  o0 = __byte_perm(a, b, 0x6420);
  o1 = __byte_perm(a, b, 0x7531);
}

// 8 neighbouring rows' sums of one token (16-byte aligned in shared memory): epilogue and store.
template <bool EXACT>
__device__ __forceinline__ void linear_store8(const LinearParams& L, const float* sums, int64_t tok, int row0) {
  float v[8], r[8];
  load8(sums, v);
  if (row0 + 8 > L.m || !L.yvec) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (row0 + i < L.m) linear_store<EXACT>(L, v[i], tok, row0 + i);
    return;
  }
  const float xs = L.xscales ? L.xscales[tok] : 1.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] *= xs;
    if (L.bias) v[i] += L.bias[row0 + i];
    v[i] = activate<EXACT>(v[i], L.activation);
  }
  if (L.residual) {
    if (L.yf32)
      load8((const float*)L.residual + tok * L.ldr + row0, r);
    else
      load8((const __nv_bfloat16*)L.residual + tok * L.ldr + row0, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += r[i];
  }
  if (L.yf32)
    store8((float*)L.y + tok * L.ldy + row0, v);
  else
    store8((__nv_bfloat16*)L.y + tok * L.ldy + row0, v);
}

// EXACT: with the activations that fp32 results want.  A kernel of its own: beside the short
// ones in one kernel they cost every call 8 to 12% (4096 x 28672 x 8192 in bf16 1.25 -> 1.35 ms).
template <class S, bool EXACT>
__global__ void __launch_bounds__(S::THREADS, 1)
    k_linear_tc(const __grid_constant__ CUtensorMap xmap, const TcParams P) {
  extern __shared__ __align__(1024) unsigned char tc_smem[];
  unsigned char* xring = (unsigned char*)(((uintptr_t)tc_smem + 1023) & ~(uintptr_t)1023);
  unsigned char* wring = xring + 2 * S::NX * S::BOX;
  float* stage = (float*)(wring + S::NW * S::WS);
  unsigned char* gring = (unsigned char*)stage + S::STAGE_BYTES;
  uint64_t* bars = (uint64_t*)(gring + S::NG * S::GS);
  // full: xF tokens, wF codes, aF expanded codes, cF sums, gF grids; free again: sD tokens and
  // expanded codes of a stage, wE codes, cE sums, gE grids
  uint64_t *xF = bars, *sD = xF + S::NX, *wF = sD + S::ND, *wE = wF + S::NW, *aF = wE + S::NW, *cF = aF + S::NA,
           *cE = cF + S::NACC, *gF = cE + S::NACC, *gE = gF + S::NG, *done = gE + S::NG;
  uint32_t* tmem_slot = (uint32_t*)(bars + S::BARRIERS);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S::NX; ++i) mbar_init(&xF[i], 1);
    for (int i = 0; i < S::ND; ++i) mbar_init(&sD[i], 1);
    for (int i = 0; i < S::NA; ++i) mbar_init(&aF[i], 8);
    for (int i = 0; i < S::NW; ++i) mbar_init(&wF[i], 1), mbar_init(&wE[i], S::X8 ? 4 : 8);   // the teams that read it

    for (int i = 0; i < S::NACC; ++i) mbar_init(&cF[i], 1), mbar_init(&cE[i], 4 * S::EW);
    for (int i = 0; i < S::NG; ++i) mbar_init(&gF[i], 1), mbar_init(&gE[i], 4 * S::EW);
    mbar_init(done, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *tmem_slot, tmem_a = tmem + S::ACC_COLS;

  const LinearParams& L = P.L;
  const int tiles = P.row_tiles * P.token_tiles, part = blockIdx.x % P.splits;
  const int tile0 = blockIdx.x / P.splits, tile_step = gridDim.x / P.splits;
  const int kb0 = part * P.per, kb1 = max(kb0, min(L.kblocks, kb0 + P.per));
  const int stages = ceil_div(kb1 - kb0, S::BPS);     // of a tile
  const long long drain = 4000000000LL;   // ~2 s: wind-down bound
  auto place = [&](int tile, int& rt, int& tt) {
    const int group = tile / (P.row_tiles * TOKEN_GROUP), in = tile - group * P.row_tiles * TOKEN_GROUP;
    const int wide = min(TOKEN_GROUP, P.token_tiles - group * TOKEN_GROUP);
    rt = in / wide;
    tt = group * TOKEN_GROUP + in % wide;
  };
  auto timed_out = [&]() {
    pdl_wait();        // the status is cleared by the kernel before
    if (!*abort_flag) raise_status(P.L.status, BAKRON_ERR_TIMEOUT);
    *abort_flag = 1;
  };
  auto wait2 = [&](uint64_t* bar, uint32_t parity, uint64_t* bar2, uint32_t parity2) {      // a warp
    if (tc_wait(bar, parity, bar2, parity2, P.spin_cycles, abort_flag)) return true;
    timed_out();
    return false;
  };
  auto wait = [&](uint64_t* bar, uint32_t parity) { return wait2(bar, parity, bar, parity); };
  auto wait_stage = [&](int it) { return wait(&sD[it % S::ND], (uint32_t)(it / S::ND) & 1u); };
  const uint32_t lead = lane == 0;
  if (warp < 4) {
    if constexpr (S::SPLIT_REGS) regs_down<S::R_LOAD>();
    if (warp == 0) {
      pdl_wait();      // the tokens' copy
      int it = 0;
      bool ok = true;
      for (int tile = tile0; tile < tiles && ok; tile += tile_step) {
        int rt, tt;
        place(tile, rt, tt);
        for (int st = 0; st < stages; ++st, ++it) {
          const int s = it % S::NX;
          if (it >= S::NX && !wait_stage(it - S::NX)) {
            ok = false;
            break;
          }
          if (lead) {
            // the second box, unless it belongs to the next part (or to nobody)
            const int col = (kb0 + st * S::BPS) * LIN_BLOCK;
            const bool two = !S::X8 || kb0 + st * 2 + 1 < kb1;
            unsigned char* to = xring + 2 * s * S::BOX;
            mbar_expect_tx(&xF[s], two ? 2 * S::BOX : S::BOX);
            tma_load_2d(to, &xmap, &xF[s], col, tt * S::BN);
            if (two) tma_load_2d(to + S::BOX, &xmap, &xF[s], col + (S::X8 ? 128 : 64), tt * S::BN);
          }
          __syncwarp();
        }
      }
      // every copy issued has landed before the CTA (and its shared memory) goes
      for (int j = it > S::NX ? it - S::NX : 0; j < it; ++j)
        if (!mbar_wait(&xF[j % S::NX], (uint32_t)(j / S::NX) & 1u, drain)) timed_out();
    } else if (warp == 2) {
      int it = 0;
      bool ok = true;
      for (int tile = tile0; tile < tiles && ok; tile += tile_step) {
        int rt, tt;
        place(tile, rt, tt);
        const unsigned char* src = L.codes + (int64_t)rt * L.kblocks * S::WS;
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
          const int s = it % S::NW;
          if (it >= S::NW && !wait(&wE[s], (uint32_t)(it / S::NW - 1) & 1u)) {
            ok = false;
            break;
          }
          if (lead) {
            mbar_expect_tx(&wF[s], S::WS);
            bulk_load(wring + s * S::WS, src + (int64_t)kb * S::WS, S::WS, &wF[s]);
          }
          __syncwarp();
        }
      }
      for (int j = it > S::NW ? it - S::NW : 0; j < it; ++j)
        if (!mbar_wait(&wF[j % S::NW], (uint32_t)(j / S::NW) & 1u, drain)) timed_out();
    } else if (warp == 3) {
      int it = 0;
      bool ok = true;
      for (int tile = tile0; tile < tiles && ok; tile += tile_step) {
        int rt, tt;
        place(tile, rt, tt);
        Segments seg(P, kb0 * 4);
        // one for each segment, or one for the tile
        for (int chunk = kb0 * 4; chunk < kb1 * 4; ++it) {
          const int s = it % S::NG, grid = L.G == 1 ? 0 : seg.seg;
          if (it >= S::NG && !wait(&gE[s], (uint32_t)(it / S::NG - 1) & 1u)) {
            ok = false;
            break;
          }
          if (lead) {
            unsigned char* to = gring + s * S::GS;
            mbar_expect_tx(&gF[s], S::GS);
            const int64_t at = grid * L.mp + (int64_t)rt * LIN_BLOCK;
            bulk_load(to, L.scales + at, S::GS, &gF[s]);
          }
          __syncwarp();
          if (L.G == 1 || seg.left == INT_MAX) {
            ++it;
            break;
          }
          chunk += seg.left;
          seg.next();
        }
      }
      for (int j = it > S::NG ? it - S::NG : 0; j < it; ++j)
        if (!mbar_wait(&gF[j % S::NG], (uint32_t)(j / S::NG) & 1u, drain)) timed_out();
    } else if (warp == 1) {
      // The warp goes through the loop together and an elected lane issues.  Cycles an MMA
      // (128 x 32, four a stage with two barrier tests, fence and commit) beside warps busy
      // on the same schedulers: elected 96, one lane all the way 117, predicated 194.
      constexpr uint32_t idesc = S::X8 ? idesc_e4m3(S::BN) : idesc_bf16(128, S::BN);
      const uint64_t desc0 = smem_desc(smem_u32(xring));
      int g = 0;
      uint32_t xs = 0, xp = 0, as = 0, ap = 0, ds = 0;     // slots and parities of the stage
      bool ok = true, here = false;
      auto sum_free = [&]() {     // before the first MMA of a segment
        return g < S::NACC || wait(&cE[g & (S::NACC - 1)], (uint32_t)(g / S::NACC - 1) & 1u);
      };
      for (int tile = tile0; tile < tiles && ok; tile += tile_step) {
        Segments seg(P, kb0 * 4);
        uint32_t more = 0;       // the segment has begun
        for (int st = 0; st < stages; ++st) {
          if (!here && (!wait2(&xF[xs], xp, &aF[as], ap) || (!more && !sum_free()))) {
            ok = false;
            break;
          }
          const uint32_t nxs = xs + 1 == S::NX ? 0 : xs + 1, nas = as + 1 == S::NA ? 0 : as + 1;
          const uint32_t nxp = xp ^ (uint32_t)(nxs == 0), nap = ap ^ (uint32_t)(nas == 0);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint64_t b = desc0 + (uint64_t)(xs * (2 * S::BOX >> 4));
          const uint32_t a = tmem_a + as * 64;
          // MMA k of the stage: 8 TMEM columns of A, 32 bytes of the tokens' rows in box k / 4
          const int nk = !S::X8 || kb0 + st * 2 + 1 < kb1 ? 8 : 4;
          if (nk == 8 && seg.left >= 8 / S::MPC) {       // no segment ends inside the stage
            if (seg.left != INT_MAX) seg.left -= 8 / S::MPC;
            const bool ends = seg.left == 0 || st == stages - 1;
            const uint32_t d = tmem + (g & (S::NACC - 1)) * S::BN;
            if (elected()) {
#pragma unroll
              for (int k = 0; k < 8; ++k)
                mma_ts<S::X8>(d, a + 8 * k, b + (k / 4) * (S::BOX >> 4) + 2 * (k % 4), idesc, k ? 1u : more);
              mma_commit(&sD[ds]);
              if (ends) mma_commit(&cF[g & (S::NACC - 1)]);
            }
            __syncwarp();
            more = 1;
            if (ends) {
              ++g;
              more = 0;
              seg.next();
            }
          } else {
#pragma unroll 1
            for (int k = 0; k < nk && ok;) {
              if (!more && k > 0) {
                ok = sum_free();
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
              }
              const int room = min(nk, (k / 4 + 1) * 4) - k;      // of this box
              const int run = seg.left < room / S::MPC ? seg.left * S::MPC : room;
              if (seg.left != INT_MAX) seg.left -= run / S::MPC;
              const bool ends = seg.left == 0 || (st == stages - 1 && k + run == nk);
              const uint32_t d = tmem + (g & (S::NACC - 1)) * S::BN;
              if (elected()) {
                const uint64_t bk = b + (k / 4) * (S::BOX >> 4);
                if (run == 4 && k % 4 == 0 && ok) {     // a box
#pragma unroll
                  for (int j = 0; j < 4; ++j) mma_ts<S::X8>(d, a + 8 * (k + j), bk + 2 * j, idesc, j ? 1u : more);
                } else {
                  for (int j = k; ok && j < k + run; ++j)
                    mma_ts<S::X8>(d, a + 8 * j, b + (j / 4) * (S::BOX >> 4) + 2 * (j % 4), idesc, j > k ? 1u : more);
                }
                if (k + run == nk) mma_commit(&sD[ds]);
                if (ends) mma_commit(&cF[g & (S::NACC - 1)]);
              }
              __syncwarp();
              k += run;
              more = 1;
              if (ends) {
                ++g;
                more = 0;
                seg.next();
              }
            }
          }
          // A look at what the next stage waits for, while the last MMAs run: most often it is
          // all there, and nothing is waited for one by one.
          const bool nx = mbar_look(&xF[nxs], nxp), na = mbar_look(&aF[nas], nap);
          const bool ns = more || g < S::NACC || mbar_look(&cE[g & (S::NACC - 1)], (uint32_t)(g / S::NACC - 1) & 1u);
          here = __all_sync(0xffffffffu, nx && na && ns);
          xs = nxs;
          xp = nxp;
          as = nas;
          ap = nap;
          ds = (ds + 1) & (S::ND - 1);
          if (!ok) break;
        }
      }
      if (elected()) mma_commit(done);
      __syncwarp();
      if (!mbar_wait(done, 0, drain)) timed_out();   // before anyone frees TMEM
    }
    __syncwarp();
  } else if (warp < 12) {
    if constexpr (S::SPLIT_REGS) regs_down<S::R_EXPAND>();
    const int row = (warp & 3) * 32 + lane, team = (warp - 4) >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    int ib = 0, ia = 0;      // blocks and stages so far
    bool ok = true;
    for (int tile = tile0; tile < tiles && ok; tile += tile_step) {
      int rt, tt;
      place(tile, rt, tt);
      const uint8_t* zeros = L.zeros + (int64_t)rt * LIN_BLOCK + row;
      auto zero_of = [&](int chunk) -> uint32_t {
        const int grid = L.G == 1 ? 0 : min(P.by_chunks ? (int)__umulhi(chunk, P.by_chunks) : chunk, L.G - 1);
        return zeros[grid * L.mp];
      };
      // the zeros of this team's chunks of a stage, two (four of e4m3 stages), asked for a load's way
      // from memory ahead (four blocks, two of e4m3 stages) and not looked at before.  (In one array
      // of two dimensions the bf16 forms were 1 to 3% slower.)
      constexpr int AHEAD = S::X8 ? 1 : 4;
      uint32_t z0[AHEAD], z1[AHEAD], z2 = 0, z3 = 0;
      auto zeros_of = [&](int kb, int i) {
        const int block = S::X8 ? kb + team : kb, chunk = block * 4 + (S::X8 ? 0 : 2 * team);
        z0[i] = z1[i] = 0;
        if (block >= kb1) return;
        z0[i] = zero_of(chunk);
        z1[i] = zero_of(chunk + 1);
        if (S::X8) z2 = zero_of(chunk + 2), z3 = zero_of(chunk + 3);
      };
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) zeros_of(i == 0 || L.G > 1 ? kb0 + i * S::BPS : kb1, i);
      for (int kb = kb0; kb < kb1; kb += S::BPS, ib += S::BPS, ++ia) {
        const uint32_t z[4] = {z0[0], z1[0], z2, z3};
        if (L.G > 1) {
#pragma unroll
          for (int i = 0; i < AHEAD - 1; ++i) z0[i] = z0[i + 1], z1[i] = z1[i + 1];
          zeros_of(kb + AHEAD * S::BPS, AHEAD - 1);
        }
        const int block = S::X8 ? ib + team : ib, sw = block % S::NW, sa = ia % S::NA;
        if (S::X8 && kb + team >= kb1) {
          // Half a stage: nothing for this team, but its arrival is this stage's, and may not come
          // while the slot still counts those of the stage NA before.
          if (ia >= S::NA && !wait_stage(ia - S::NA)) {
            ok = false;
            break;
          }
          __syncwarp();
          if (lead) mbar_arrive(&aF[sa]);
          continue;
        }
        if (!wait(&wF[sw], (uint32_t)(block / S::NW) & 1u) || (ia >= S::NA && !wait_stage(ia - S::NA))) {
          ok = false;
          break;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint4* u = reinterpret_cast<const uint4*>(wring + sw * S::WS) + row;
        const uint32_t to = tmem_a + sa * 64 + team * 32 + lanes;
        uint32_t a[16];
        if constexpr (S::X8) {
          uint4 q[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) q[t] = u[t * 128];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
              minus_zero8(j == 0 ? q[t].x : j == 1 ? q[t].y : j == 2 ? q[t].z : q[t].w, z[j] * 0x01010101u,
                          a[8 * (j & 1) + 2 * t], a[8 * (j & 1) + 2 * t + 1]);
            if (j & 1) tmem_st16(to + 8 * (j - 1), a);
          }
        } else if constexpr (S::W8) {
          uint4 q[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) q[t] = u[(t + 4 * team) * 128];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const __nv_bfloat162 zz = __float2bfloat162_rn((float)z[j]);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
              for (int p = 0; p < 4; ++p) a[4 * t + p] = pair8(j ? q[t].z : q[t].x, j ? q[t].w : q[t].y, p, zz);
            tmem_st16(to + 16 * j, a);
          }
        } else {
          uint2 q[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) q[t] = reinterpret_cast<const uint2*>(u + t * 128)[team];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const __nv_bfloat162 zz = __float2bfloat162_rn((float)z[j] + 128.f);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
              for (int p = 0; p < 4; ++p) a[4 * t + p] = pair4(j ? q[t].y : q[t].x, p, zz);
            tmem_st16(to + 16 * j, a);
          }
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lead) {
          mbar_arrive(&aF[sa]);
          mbar_arrive(&wE[sw]);
        }
      }
      if (S::X8 && ((kb1 - kb0) & 1)) --ib;      // the half stage had one block
    }
  } else {
    if constexpr (S::SPLIT_REGS) regs_up<S::R_SUM>();
    const int q = warp & 3, ch = (warp - 12) >> 2;      // lane quarter, part of the columns
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    int g = 0, ig = 0;
    bool ok = true;
    for (int tile = tile0; tile < tiles && ok; tile += tile_step) {
      int rt, tt;
      place(tile, rt, tt);
      Two acc[S::COLS / 2];       // in pairs: half the instructions (issue slots are what is short)
#pragma unroll
      for (int i = 0; i < S::COLS / 2; ++i) acc[i] = Two(0.f, 0.f);
      Segments seg(P, kb0 * 4);
      float s = 0.f;
      for (int chunk = kb0 * 4; chunk < kb1 * 4; ++g) {
        const int buf = g & (S::NACC - 1);
        const bool fresh = L.G > 1 || chunk == kb0 * 4;       // the next grid
        uint64_t* gbar = &gF[ig % S::NG];
        if (!(fresh ? wait2(&cF[buf], (uint32_t)(g / S::NACC) & 1u, gbar, (uint32_t)(ig / S::NG) & 1u)
                    : wait(&cF[buf], (uint32_t)(g / S::NACC) & 1u))) {
          ok = false;
          break;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (fresh) {
          s = reinterpret_cast<const float*>(gring + (ig % S::NG) * S::GS)[q * 32 + lane] * (S::X8 ? 512.f : 1.f);
        }
        // As much of the sums at once as registers allow: a warp's turn is a chain of waits.
        const uint32_t at = tmem + lanes + buf * S::BN + ch * S::COLS;
        constexpr int LD = S::COLS <= 64 ? S::COLS : 32;
#pragma unroll
        for (int c = 0; c < S::COLS; c += LD) {
          uint32_t r[LD / 16][16];
#pragma unroll
          for (int i = 0; i < LD / 16; ++i) tmem_ld16(at + c + 16 * i, r[i]);
          tmem_wait_ld();
          if (c + LD == S::COLS) {      // all read: the next segment's MMAs may have it
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lead) mbar_arrive(&cE[buf]);
          }
#pragma unroll
          for (int i = 0; i < LD; i += 2)
            acc[(c + i) / 2] = Two::fma(Two(s, s), Two(__uint_as_float(r[i / 16][i % 16]), __uint_as_float(r[i / 16][i % 16 + 1])),
                                        acc[(c + i) / 2]);
        }
        chunk = seg.left == INT_MAX ? INT_MAX : chunk + seg.left;
        seg.next();
        if (L.G > 1 || chunk >= kb1 * 4) {
          __syncwarp();
          if (lead) mbar_arrive(&gE[ig % S::NG]);
          ++ig;
        }
      }
      if (!ok) break;
      if (S::BN <= 128 && P.splits > 1) {
        // [token][128 rows] over the tokens' ring: every MMA that read it is complete
#pragma unroll
        for (int i = 0; i < S::COLS; i += 2) {
          float* to = (float*)xring + (ch * S::COLS + i) * 128 + q * 32 + lane;
          acc[i / 2].get(to[0], to[128]);
        }
      } else {
        float* mine = stage + (warp - 12) * 8 * STAGE_LD;
        const int row0 = rt * LIN_BLOCK + q * 32 + (lane & 3) * 8;
#pragma unroll 1
        for (int b = 0; b < S::COLS / 8; ++b) {
          __syncwarp();
#pragma unroll
          for (int c = 0; c < S::COLS / 8; ++c)
            if (b == c) {     // registers: no index that is not constant
#pragma unroll
              for (int i = 0; i < 8; i += 2)
                acc[4 * c + i / 2].get(mine[i * STAGE_LD + lane], mine[(i + 1) * STAGE_LD + lane]);
            }
          __syncwarp();
          const int64_t tok = (int64_t)tt * S::BN + ch * S::COLS + b * 8 + (lane >> 2);
          if (tok < L.rows) linear_store8<EXACT>(L, mine + (lane >> 2) * STAGE_LD + (lane & 3) * 8, tok, row0);
        }
      }
    }
  }
  if constexpr (S::BN <= 128) {
    if (P.splits > 1) {      // one tile a cluster; every thread of it comes here
      cg::cluster_group cluster = cg::this_cluster();
      float* mine = (float*)xring;
      cluster.sync();
      int rt, tt;
      place(tile0, rt, tt);
      const int row = rt * LIN_BLOCK + (threadIdx.x & 127);
      for (int t = part * (3 + S::EW) + (threadIdx.x >> 7); t < S::BN; t += (3 + S::EW) * P.splits) {
        const int64_t tok = (int64_t)tt * S::BN + t;
        if (tok >= L.rows) break;
        float v = 0.f;
        for (int p = 0; p < P.splits; ++p)
          v += cluster.map_shared_rank(mine, p)[t * 128 + (threadIdx.x & 127)];
        if (row < L.m) linear_store<EXACT>(L, v, tok, row);
      }
      cluster.sync();          // nobody's shared memory goes before it is read
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// Tokens as TMA can read them: rows of 16-byte multiples, e4m3 widened to bf16 (exact)
// where the codes have 8 bits.
// Clears the status, too.
template <bool X8, bool WIDEN>
__global__ void __launch_bounds__(256)
    k_linear_rows(const void* x, int64_t ldx, int n, void* out, int64_t ldo, int* status) {
  pdl_trigger();
  if (blockIdx.x + blockIdx.y + threadIdx.x == 0) *status = 0;
  const int64_t row = blockIdx.x;
  for (int k = blockIdx.y * 1024 + threadIdx.x; k < min(n, (int)(blockIdx.y + 1) * 1024); k += 256) {
    if constexpr (!X8) {
      ((uint16_t*)out)[row * ldo + k] = ((const uint16_t*)x)[row * ldx + k];
    } else {
      const uint8_t v = ((const uint8_t*)x)[row * ldx + k];
      if constexpr (WIDEN)
        ((__nv_bfloat16*)out)[row * ldo + k] =
            __float2bfloat16_rn(__half2float(__half(__nv_cvt_fp8_to_halfraw(v, __NV_E4M3))));
      else
        ((uint8_t*)out)[row * ldo + k] = v;
    }
  }
}

__global__ void k_clear_status(int* status) {
  pdl_trigger();
  *status = 0;
}

template <class S, bool EXACT>
int launch_tc(const void* x, int64_t ldx, TcParams& P, cudaStream_t s) {
  static OncePerDevice once;
  BK_CUDA_OK(once([] {
    cudaFuncAttributes a;
    cudaError_t e = cudaFuncGetAttributes(&a, k_linear_tc<S, EXACT>);
    // the warpgroups' shares (setmaxnreg) are taken from what the block is launched with
    if (e == cudaSuccess && S::SPLIT_REGS && a.numRegs != S::LAUNCH_REGS) e = cudaErrorInvalidConfiguration;
    return e != cudaSuccess
               ? e
               : cudaFuncSetAttribute(k_linear_tc<S, EXACT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::SMEM);
  }));
  const LinearParams& L = P.L;
  P.token_tiles = ceil_div(L.rows, S::BN);
  const int64_t tiles = (int64_t)P.row_tiles * P.token_tiles;
  if (tiles > INT_MAX / 16) return BAKRON_ERR_INVALID_ARG;
  P.splits = 1;
  if (S::BN <= 128)
    while (P.splits < 8 && tiles * P.splits * 2 <= ROW_SMS && L.kblocks >= 4 * P.splits) P.splits *= 2;
  P.per = ceil_div(L.kblocks, P.splits);
  CUtensorMap map;
  const cuuint64_t dims[2] = {(cuuint64_t)L.n, (cuuint64_t)L.rows};
  const cuuint64_t strides[1] = {(cuuint64_t)ldx * (S::X8 ? 1 : 2)};
  const cuuint32_t box[2] = {S::X8 ? 128u : 64u, (cuuint32_t)S::BN}, ones[2] = {1u, 1u};
  if (!get_encode() ||
      g_encode(&map, S::X8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(x), dims,
               strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return BAKRON_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(P.splits > 1 ? tiles * P.splits : std::min<int64_t>(tiles, ROW_SMS)));
  cfg.blockDim = dim3(S::THREADS);
  cfg.dynamicSmemBytes = S::SMEM;
  cfg.stream = s;
  // Starts beside the kernel before (which clears the status and makes the tokens'
  // copy): barriers, TMEM and the first codes are ready when that is done.
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = P.splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = P.splits > 1 ? 2 : 1;
  BK_CUDA_OK(cudaLaunchKernelEx(&cfg, k_linear_tc<S, EXACT>, map, P));
  return BAKRON_OK;
}

template <bool W8, bool X8, bool EXACT>
int launch_bn(const void* x, int64_t ldx, TcParams& P, cudaStream_t s) {
  // The token tile with the shortest schedule: rounds of tiles over the SMs, a tile costing
  // its tokens and about 32 more (expanding the codes, the way out).
  int best = 32;
  double cost = 1e300;
  for (int bn : {192, 128, 64, 32}) {
    const double tiles = (double)P.row_tiles * ceil_div(P.L.rows, bn);
    const double c = tiles >= ROW_SMS ? ceil(tiles / ROW_SMS) * (bn + 32) : tiles / ROW_SMS * (bn + 32) + (bn > 128 ? bn : 0);
    if (c < 0.97 * cost) {
      best = bn;
      cost = c;
    }
  }
  switch (best) {
    case 192: return launch_tc<TcShape<192, W8, X8>, EXACT>(x, ldx, P, s);
    case 128: return launch_tc<TcShape<128, W8, X8>, EXACT>(x, ldx, P, s);
    case 64: return launch_tc<TcShape<64, W8, X8>, EXACT>(x, ldx, P, s);
    default: return launch_tc<TcShape<32, W8, X8>, EXACT>(x, ldx, P, s);
  }
}

}  // namespace

// Whether TMA reads the tokens as they are; if not, they are copied first.
static bool rows_in_place(const void* x, bool x8, int64_t ldx, bool bytes8) {
  return !(x8 && bytes8) && aligned16(x, x8 ? ldx : 2 * ldx);
}

// The workspace: [status 256 B][tokens' copy].
size_t linear_tc_workspace(const void* x, bool x8, int rows, int64_t ldx, int n, bool bytes8) {
  return 256 + (rows_in_place(x, x8, ldx, bytes8) ? 0 : (size_t)rows * round_up(n, 16) * (x8 && !bytes8 ? 1 : 2));
}

int linear_tc(const LinearParams& L, bool x8, bool bytes8, void* workspace, cudaStream_t s) {
  TcParams P{};
  P.L = L;
  P.row_tiles = (int)(L.mp / LIN_BLOCK);
  P.by_chunks = L.chunks > 1 ? (uint32_t)((((uint64_t)1 << 32) + L.chunks - 1) / L.chunks) : 0;
  P.seg_chunks = L.G > 1 ? L.chunks : x8 && !bytes8 ? SEG_MMAS : SEG_MMAS / 2;
  P.segs = L.G > 1 ? L.G : INT_MAX / SEG_MMAS - 1;
  P.spin_cycles = spin_cycles_from_env();
  const void* x = L.x;
  int64_t ldx = L.ldx;
  if (!rows_in_place(x, x8, ldx, bytes8)) {
    void* out = (char*)workspace + 256;
    const dim3 grid((unsigned)L.rows, (unsigned)ceil_div(L.n, 1024));
    ldx = round_up(L.n, 16);
    if (!x8)
      k_linear_rows<false, false><<<grid, 256, 0, s>>>(x, L.ldx, L.n, out, ldx, L.status);
    else if (bytes8)
      k_linear_rows<true, true><<<grid, 256, 0, s>>>(x, L.ldx, L.n, out, ldx, L.status);
    else
      k_linear_rows<true, false><<<grid, 256, 0, s>>>(x, L.ldx, L.n, out, ldx, L.status);
    BK_CUDA_OK(cudaGetLastError());
    x = out;
  } else {
    k_clear_status<<<1, 1, 0, s>>>(L.status);
    BK_CUDA_OK(cudaGetLastError());
  }
  const bool exact = exact_activation(L);
  if (bytes8) return exact ? launch_bn<true, false, true>(x, ldx, P, s) : launch_bn<true, false, false>(x, ldx, P, s);
  if (x8) return exact ? launch_bn<false, true, true>(x, ldx, P, s) : launch_bn<false, true, false>(x, ldx, P, s);
  return exact ? launch_bn<false, false, true>(x, ldx, P, s) : launch_bn<false, false, false>(x, ldx, P, s);
}

}  // namespace bakron
