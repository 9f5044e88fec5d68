// bakron_linear_backward: dx = dy What, the gradient of y = x What^T at the tokens x,
// What_ij = s (c_ij - z) with the grid (s, z) of row i and j's group.
//
// The sum runs over What's rows, whose scales differ, so the scale cannot wait for the end of a
// sum as it does in the forward product: it multiplies an operand.
//
// Up to 8 tokens: mma.sync on operands formed in registers, c - z (exact) and dy s in two bf16 parts.  More: s (c - z) is
// formed in fp16, whose 11 bits leave the result's rounding to bf16's 8 the only one that counts, and dy is
// exact there: a token's gradients are multiplied by the power of two that takes its largest one to 2^15 (32 binades below it
// lose no bit, and what is lost further down is 2^-40 of it), the scales by the one that takes the weight's largest to
// 2^6; the result is multiplied back.
//
// Few: D (128 columns of What x bn tokens) += A B on the 5th-generation tensor cores with A the
// operands of a 128 x 128 block, formed from its codes in shared memory as the MMAs take them (MN-major), and B the
// tokens' gradients, K-major by TMA.  Many: the weight is written out in fp16 once, and read by the pair product.
//
// us, caches flushed: 1 token, groups of 128, 4096 x 4096 12, 28672 x 8192 55 (2.4 TB/s with the scales); 17 tokens through
// 4099 x 11003 in 8 bits 27; 64 through 11008 x 4096 28, 256 48, 4096 275 (1.34 PFLOP/s; 20 of them to write the weight out, 26
// the tokens).  In bf16, with an error 1.35 times the result's rounding, dy needs no pass of its own: 25, 43, 240.
#include <float.h>

#include <cuda_fp16.h>

#include <algorithm>

#include "linear.cuh"
#include "pair_gemm.cuh"

namespace bakron {
namespace {

// ------------------------------------------------------------------ operands
constexpr int FB_WARPS = 16;                     // form operands
constexpr int FB_THREADS = 32 * (8 + FB_WARPS);  // warps 0 and 2 load, warp 1 issues MMAs, warps 4-7 write out
constexpr uint32_t FB_A = LIN_BLOCK * LIN_BLOCK * 2;   // operands: [64 rows][64 columns], two by two
constexpr int FB_RING = 8;                       // most stages of a ring
constexpr int FB_MAX_BN = 192;
constexpr int FB_GROUP = 32;                     // blocks summed in place: 4096 products (pair_gemm.cuh says why)

struct FusedParams {
  const unsigned char* codes;
  const float* scales;
  const uint8_t* zeros;
  int64_t mp;
  int kblocks, chunks, G;
  int rows, n, bn;         // tokens, columns, tokens of a tile (a multiple of 16)
  int nk, token_tiles, tiles;      // 128-row blocks; tiles in all
  int na, nb, nc;          // stages of the operands' ring, the gradients', the codes'
  const int* top;          // the largest scale's exponent
  const float2* power;     // a token's power of two
  __nv_bfloat16* dx;
  int64_t ldx;
  float* part;             // [CTA][its first tile, its last][token][128 columns]
  int vec;                 // dx can be written 8 bytes at a time
  int* status;             // and each CTA's error or 0, which the last kernel joins
  int* flags;
  long long spin_cycles;
};

// The CTAs' equal shares of all tiles' blocks.
struct Shares {
  int64_t units;
  int nk, ctas;
  __host__ __device__ Shares(const FusedParams& P, int ctas_) : units((int64_t)P.tiles * P.nk), nk(P.nk), ctas(ctas_) {}
  __host__ __device__ __forceinline__ int64_t begin(int cta) const { return units * cta / ctas; }
  __host__ __device__ int owner(int64_t unit) const {
    int i = (int)(unit * ctas / units);
    while (begin(i + 1) <= unit) ++i;
    return i;
  }
  // of a CTA's sums of a tile: its first tile, or another (then its last)
  __host__ __device__ __forceinline__ int64_t slot(int cta, int tile) const { return 2 * (int64_t)cta + (begin(cta) / nk != tile); }
};

// Scales are multiplied by 2^of(exponent field of the weight's largest), which takes that one to [2^6, 2^7), so that
// s (c - z) stays below 2^15.
__host__ __device__ constexpr int scale_power(int top) { return top < 6 ? 127 : 133 - top; }
__device__ __forceinline__ float scale_factor(const int* top) { return __uint_as_float((uint32_t)(scale_power(__ldg(top)) + 127) << 23); }

// A row's grid: two codes' values in fp16 are (c - z) hi + (c - z) lo, s = hi + lo to 2^-22, rounded once (the small
// product's own rounding is 2^-22 of it).
struct RowGrid {
  uint32_t z;      // 1024 + z, twice
  __half2 hi, lo;
  __device__ __forceinline__ void set(float s, uint32_t zero) {
    z = zero * 0x00010001u + 0x64006400u;
    hi = __float2half2_rn(s);
    lo = __float2half2_rn(s - __low2float(hi));
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t codes1024) const {      // 1024 + c, exact
    const __half2 c = __hsub2(*reinterpret_cast<const __half2*>(&codes1024), *reinterpret_cast<const __half2*>(&z));
    const __half2 r = __hfma2(c, hi, __hmul2(c, lo));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
};
// Pair p of chunk j (32 columns, 8 of them a unit's) of a unit: columns 2p, 2p + 1 of its 8.
__device__ __forceinline__ uint32_t operand4(uint32_t word, int p, const RowGrid& g) {
  return g(((word >> (4 * p)) & 0x000F000Fu) | 0x64006400u);
}
__device__ __forceinline__ uint32_t operand8(uint32_t word, int odd, const RowGrid& g) {
  return g(__byte_perm(word, 0x64646464u, odd ? 0x4341 : 0x4240));
}
__device__ __forceinline__ uint32_t operand(const uint4 (&u)[1], int j, int p, const RowGrid& g) {
  return operand4(reinterpret_cast<const uint32_t*>(&u[0])[j], p, g);
}
__device__ __forceinline__ uint32_t operand(const uint4 (&u)[2], int j, int p, const RowGrid& g) {
  return operand8(reinterpret_cast<const uint32_t*>(&u[j >> 1])[2 * (j & 1) + (p >> 1)], p & 1, g);
}

// A token's gradients in fp16: times 2^k, k from the largest finite one, exact from 2^-32 of it on.  power: what takes the
// product's sums back.  The token's row is read twice, the second time from the caches.
template <bool VEC>
__global__ void __launch_bounds__(512) k_back_tokens(const __nv_bfloat16* from, int64_t ld, int m, const int* top, __half* to,
                                                     int64_t ldt, float2* power, int* status) {
  __shared__ uint32_t slots[16];
  pdl_trigger();      // the product may get ready; it waits for this grid's end
  const int64_t row = blockIdx.x;
  const uint16_t* in = reinterpret_cast<const uint16_t*>(from) + row * ld;
  __half* out = to + row * ldt;
  const int whole = VEC ? m & ~7 : 0;
  uint32_t most = 0;      // the largest magnitude's bits
  auto look = [&](uint32_t v) {
    v &= 0x7fffu;
    most = max(most, v < 0x7f80u ? v : 0u);
  };
#pragma unroll 4
  for (int c = threadIdx.x * 8; c < whole; c += 4096) {
    const uint4 u = *reinterpret_cast<const uint4*>(in + c);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      look(w[j]);
      look(w[j] >> 16);
    }
  }
#pragma unroll 4
  for (int c = whole + threadIdx.x; c < m; c += 512) look(in[c]);
  most = __reduce_max_sync(0xffffffffu, most);
  if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = most;
  __syncthreads();
  most = __reduce_max_sync(0xffffffffu, slots[threadIdx.x & 15]);
  const int k = most ? 141 - max((int)(most >> 7), 1) : 0;      // below 2^(field - 126): to below 2^15
  if (threadIdx.x == 0) {
    power[row] = two_powers(-k - scale_power(__ldg(top)));
    if (row == 0 && status) *status = 0;
  }
  const float2 scale = two_powers(k);
  auto half = [&](uint32_t bits) { return times(__uint_as_float(bits), scale); };
#pragma unroll 4
  for (int c = threadIdx.x * 8; c < whole; c += 4096) {
    const uint4 u = *reinterpret_cast<const uint4*>(in + c);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const __half2 v = __floats2half2_rn(half(w[j] << 16), half(w[j] & 0xffff0000u));
      o[j] = *reinterpret_cast<const uint32_t*>(&v);
    }
    *reinterpret_cast<uint4*>(out + c) = make_uint4(o[0], o[1], o[2], o[3]);
  }
#pragma unroll 4
  for (int c = whole + threadIdx.x; c < m; c += 512) out[c] = __float2half_rn(half((uint32_t)in[c] << 16));
}

// ------------------------------------------------------------------ up to 8 tokens
// No tensor memory, no shared operands: mma.sync takes What's columns as the rows of its first operand
// and What's rows as its depth.  A warp has a column block and 16 rows at a time: lane group g unit g & 3 of
// them (32 columns of a row), and of each word's 8 columns the four that g >> 2 says; lane q of it rows
// 4q..4q+3, so that two rows' columns become, halves exchanged, operand registers of 2 products.  The order of the
// 16 rows is free: the tokens' values (its second operand) are those of rows 4q..4q+3.
//
// The first operand is c - z, an integer of 8 bits.  The scale goes to the tokens' side, where a lane has 4 values
// instead of 64, and the 16 columns of a product have one grid: dy s = hi + lo, two bf16 numbers that keep it to
// 2^-15, so that the result's rounding is all that counts (s (c - z) rounded to bf16 made the error 1.4 times that and
// more).  Up to 4 tokens hi and lo are columns of one product, g and g + 4, added at the end; up to 8 a product each.
//
// 1 token x 28672 x 8192 55 us, 8 tokens 57: neither products nor codes bound it (twice the products cost nothing), but the
// way of the codes into registers (2.1 TB/s; through shared memory, 4 stages a warp, 58 and 63).
constexpr int FEW_BACK = 8, FW_COLS = LIN_BLOCK, FW_WARPS = 8;
constexpr int FW_TOKEN = FW_COLS + 1;      // stride of the warps' sums
constexpr int FW_SMEM = FW_WARPS * FEW_BACK * FW_TOKEN * 4;
constexpr int few_ahead(bool w8, bool one) { return w8 || !one ? 1 : 2; }      // chunks of a warp on their way
constexpr int few_ctas(bool w8, bool one) { return w8 && !one ? 1 : 2; }      // an SM holds, by their registers

__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                            uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

struct FewParams {
  const unsigned char* codes;
  const float* scales;
  const uint8_t* zeros;
  int64_t mp;
  int kblocks, chunks, G;
  int rows, m, n, chunks16, per;      // 16-row chunks in all, of a CTA (a multiple of 8)
  const __nv_bfloat16* dy;
  int64_t lddy;
  int yvec;                           // dy can be read 8 bytes at a time, and m is a multiple of 4
  float* part;                        // [split][token][column tiles' 256]
  int* status;
};

// Two rows' codes of a chunk as c - z in bf16, in the products' order: o[0..1] the first columns of the pairs
// p = 2 upper + k, o[2..3] their second ones, each register one column of the two rows.  A word is
// transposed by its bytes first: a pair's columns lie in its bytes `upper` and 2 + `upper` (4 bits), or k and 2 + k.
// zeros: a byte a row.
template <bool W8>
__device__ __forceinline__ void integers(uint32_t w0, uint32_t w1, bool upper, uint32_t zeros, int row, uint32_t (&o)[4]) {
  if constexpr (W8) {      // 1024 + c in fp16, exact
    const uint32_t z = __byte_perm(zeros, 0x64646464u, row | 0x4040 | (row + 1) << 8);
    const uint32_t t[2] = {__byte_perm(w0, w1, 0x5140), __byte_perm(w0, w1, 0x7362)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t v = __byte_perm(t[i >> 1], 0x64646464u, i & 1 ? 0x4342 : 0x4140);
      const float2 c = __half22float2(__hsub2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&z)));
      o[i] = bf16_pack(c.x, c.y);
    }
  } else {      // 128 + c in bf16
    const uint32_t z = __byte_perm(zeros, 0x43434343u, row | 0x4040 | (row + 1) << 8);
    const uint32_t t[2] = {__byte_perm(w0, w1, upper ? 0x0501 : 0x0400), __byte_perm(w0, w1, upper ? 0x0703 : 0x0602)};
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = pair4(t[i >> 1], i & 1, *reinterpret_cast<const __nv_bfloat162*>(&z));
  }
}
// v = hi + lo: hi its leading 8 bits, lo the rest, rounded.  An infinity is all hi.
__device__ __forceinline__ void two_parts(const float (&v)[4], uint32_t (&hi)[2], uint32_t (&lo)[2]) {
  float r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = v[i] - __uint_as_float(__float_as_uint(v[i]) & 0xffff0000u);
  if (fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3]))) > FLT_MAX) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = fabsf(v[i]) > FLT_MAX ? 0.f : r[i];
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    hi[i] = __byte_perm(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]), 0x7632);
    lo[i] = bf16_pack(r[2 * i], r[2 * i + 1]);
  }
}

// ONE: the 128 columns of a block have one grid a row.  FOUR: up to 4 tokens.  VEC: dy can be read 8 bytes at a time, and
// m is a multiple of 4.  (No load stands behind a branch: a value that two ways lead to is waited for where they meet.)
template <bool W8, bool ONE, bool FOUR, bool VEC>
__global__ void __launch_bounds__(FW_WARPS * 32, few_ctas(W8, ONE)) k_back_few(const FewParams P) {
  constexpr int UNITS = W8 ? 8 : 4, H = W8 ? 2 : 1, GRIDS = ONE ? 1 : 4;
  extern __shared__ float fw_sums[];      // [warp][column of the products][What's column]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int cb = blockIdx.x, t = g & 3, token = FOUR ? t : g;
  const bool upper = g >> 2;
  if (blockIdx.x + blockIdx.y + threadIdx.x == 0) *P.status = 0;      // nothing here can run out
  const int first = blockIdx.y * P.per, last = min(first + P.per, P.chunks16);
  int grid[GRIDS];
#pragma unroll
  for (int j = 0; j < GRIDS; ++j) grid[j] = P.G == 1 ? 0 : min((cb * 4 + j) / P.chunks, P.G - 1);
  struct Chunk {
    uint4 u[4][H];
    float4 s[GRIDS];
    uint32_t z[GRIDS];
    uint32_t y[VEC ? 2 : 4];
  };
  const __nv_bfloat16* dy = P.dy + min(token, P.rows - 1) * P.lddy;
  auto load = [&](int chunk, Chunk& to) {
    const int row = chunk * 16 + 4 * q;
    const uint4* at = reinterpret_cast<const uint4*>(P.codes) +
                      (((int64_t)(row >> 7) * P.kblocks + cb) * UNITS + t) * LIN_BLOCK + (row & 127);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int h = 0; h < H; ++h) to.u[r][h] = __ldg(at + h * 4 * LIN_BLOCK + r);
#pragma unroll
    for (int j = 0; j < GRIDS; ++j) {
      to.s[j] = __ldg(reinterpret_cast<const float4*>(P.scales + grid[j] * P.mp + row));
      to.z[j] = __ldg(reinterpret_cast<const uint32_t*>(P.zeros + grid[j] * P.mp + row));
    }
    if constexpr (VEC) {
      const uint2 v = __ldg(reinterpret_cast<const uint2*>(dy + min(row, P.m - 4)));
      to.y[0] = v.x;
      to.y[1] = v.y;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) to.y[k] = __ldg(reinterpret_cast<const unsigned short*>(dy) + min(row + k, P.m - 1));
    }
  };
  float acc[8][4] = {};
  auto products = [&](const Chunk& here, int chunk) {
    uint32_t hi[2], lo[2];
    float y[4];      // 0 for no token, and behind the last row
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t v = VEC ? (k & 1 ? here.y[k >> 1] & 0xffff0000u : here.y[k >> 1] << 16) : here.y[k] << 16;
      y[k] = token < P.rows && chunk * 16 + 4 * q + k < P.m ? __uint_as_float(v) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j < GRIDS) {
        const float4 s = here.s[j];
        const float v[4] = {y[0] * s.x, y[1] * s.y, y[2] * s.z, y[3] * s.w};
        two_parts(v, hi, lo);
        if (FOUR && upper) hi[0] = lo[0], hi[1] = lo[1];
      }
      uint32_t a[4], b[4];      // rows 4q, 4q + 1; 4q + 2, 4q + 3
      auto word = [&](int r) -> uint32_t {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(here.u[r]);
        return W8 ? (upper ? w[2 * j + 1] : w[2 * j]) : w[j];
      };
      integers<W8>(word(0), word(1), upper, here.z[j < GRIDS ? j : 0], 0, a);
      integers<W8>(word(2), word(3), upper, here.z[j < GRIDS ? j : 0], 2, b);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        mma_16x8x16(acc[2 * j + k], a[k], a[2 + k], b[k], b[2 + k], hi[0], hi[1]);
        if (!FOUR) mma_16x8x16(acc[2 * j + k], a[k], a[2 + k], b[k], b[2 + k], lo[0], lo[1]);
      }
    }
  };
  constexpr int AHEAD = few_ahead(W8, ONE);
  Chunk next[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (first + warp + i * FW_WARPS < last) load(first + warp + i * FW_WARPS, next[i]);
  for (int chunk = first + warp; chunk < last; chunk += AHEAD * FW_WARPS) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int c = chunk + i * FW_WARPS;
      if (i > 0 && c >= last) break;
      const Chunk here = next[i];
      if (c + AHEAD * FW_WARPS < last) load(c + AHEAD * FW_WARPS, next[i]);
      products(here, c);
    }
  }
  float* mine = fw_sums + warp * FEW_BACK * FW_TOKEN + 8 * t + (upper ? 4 : 0);
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e)      // column of the pair e >> 1, of the products 2q + (e & 1)
      mine[(2 * q + (e & 1)) * FW_TOKEN + 32 * (i >> 1) + 2 * (i & 1) + (e >> 1)] = acc[i][e];
  __syncthreads();
  const int c = threadIdx.x % FW_COLS;
  for (int tok = threadIdx.x / FW_COLS; tok < P.rows; tok += FW_WARPS * 32 / FW_COLS) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < FW_WARPS; ++w) {
      v += fw_sums[(w * FEW_BACK + tok) * FW_TOKEN + c];
      if (FOUR) v += fw_sums[(w * FEW_BACK + tok + 4) * FW_TOKEN + c];
    }
    P.part[(((int64_t)blockIdx.y * P.rows + tok) * gridDim.x + blockIdx.x) * FW_COLS + c] = v;
  }
  pdl_trigger();
}

__global__ void __launch_bounds__(256) k_back_few_sum(const float* part, int splits, int rows, int tiles, int n,
                                                      __nv_bfloat16* dx, int64_t ldx) {
  const int col = blockIdx.x * 256 + threadIdx.x, tok = blockIdx.y;
  pdl_wait();
  if (col >= n) return;
  float v = 0.f;
#pragma unroll 8
  for (int s = 0; s < splits; ++s) v += part[((int64_t)s * rows + tok) * tiles * FW_COLS + col];
  dx[tok * ldx + col] = __float2bfloat16_rn(v);
}

// ------------------------------------------------------------------ more
// A CTA takes an equal share of all tiles' blocks, one after another; a tile that several share is
// summed from their parts, in their order, by a second kernel.  (As clusters that add
// through each other's shared memory, no more than 15 of 8 CTAs ran at a time.)
// ONE: the 128 columns of a block have one grid a row.  TEAMS: see below; na and nc are multiples of
// it, so that a ring's slot always belongs to one team, which knows the phase it is in.
//
// Bound by the issue of MMAs, some 100 cycles each however few tokens they have: the 8 of a block, its two commits
// and waits take 900 cycles (16 x 28672 x 8192 52 of 72 us with neither loads nor operands formed), the
// operands 1000 beside them.  (Tokens as the MMA's 128 rows and 256 columns of What, half as many MMAs, took 99: its
// copies are of a kilobyte, 50 cycles each.)  From 128 tokens on by the MMAs themselves.
template <bool W8, bool ONE, int TEAMS>
__global__ void __launch_bounds__(FB_THREADS, 1) k_back_fused(const __grid_constant__ CUtensorMap map, const FusedParams P) {
  constexpr int TEAM = FB_WARPS / TEAMS;      // warps
  constexpr uint32_t CODES = W8 ? 16384 : 8192, GRID = LIN_BLOCK * 5, GRIDS = ONE ? 1 : 4;
  extern __shared__ __align__(1024) unsigned char fb_smem[];
  unsigned char* smem = (unsigned char*)(((uintptr_t)fb_smem + 1023) & ~(uintptr_t)1023);
  const uint32_t half_b = (uint32_t)P.bn * 128u;
  unsigned char* tokens = smem + P.na * FB_A;     // [nb][two 64-row halves][bn][64]
  unsigned char* codes = tokens + P.nb * 2 * half_b;     // [nc][codes], then [nc][GRIDS][scales, zeros]
  unsigned char* grids = codes + P.nc * CODES;
  // F: tokens and codes loaded, operands formed, sums finished; E: free again
  __shared__ uint64_t bF[FB_RING], bE[FB_RING], cF[FB_RING], cE[FB_RING], aF[FB_RING], aE[FB_RING], accF[2], accE[2],
      done;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Shares share(P, gridDim.x);
  const int64_t u0 = share.begin(blockIdx.x), u1 = share.begin(blockIdx.x + 1);
  const int tile0 = (int)(u0 / P.nk), first_k = (int)(u0 % P.nk), count = (int)(u1 - u0);
  uint32_t cols = 32;      // of TMEM, for one tile's sums
  while (cols < (uint32_t)P.bn) cols *= 2;

  if (threadIdx.x == 0) {
    for (int i = 0; i < FB_RING; ++i) {
      mbar_init(&bF[i], 1);
      mbar_init(&bE[i], 1);
      mbar_init(&cF[i], 1);
      mbar_init(&cE[i], TEAM);
      mbar_init(&aF[i], TEAM);
      mbar_init(&aE[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&accF[i], 1);
      mbar_init(&accE[i], 4);
    }
    mbar_init(&done, 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)),
                 "r"(2 * cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  constexpr long long drain = 4000000000LL;      // about 2 s: the bound of the way out
  // a warp's wait; `out`: on the way out, whatever happened elsewhere
  auto wait = [&](uint64_t* bar, uint32_t parity, bool out = false) -> bool {
    if (mbar_wait_warp(bar, parity, out ? drain : P.spin_cycles, out ? nullptr : &abort_flag)) return true;
    if (lane == 0) abort_flag = 1;
    __syncwarp();
    return false;
  };

  if (warp == 0) {
    // ------------------------------------------------------------ gradients
    pdl_wait();      // (the codes' loads need no kernel before: the one that this waits for has waited for the rest)
    int it = 0, s = 0, k = first_k, tile = tile0;
    uint32_t parity = 1;      // a fresh barrier's phase before the first counts as complete
    for (; it < count; ++it) {
      if (!wait(&bE[s], parity)) break;
      if (elected()) {
        unsigned char* to = tokens + s * 2 * half_b;
        const int tok = tile % P.token_tiles * P.bn;
        mbar_expect_tx(&bF[s], 2 * half_b);
        tma_load_2d(to, &map, &bF[s], k * LIN_BLOCK, tok);
        tma_load_2d(to + half_b, &map, &bF[s], k * LIN_BLOCK + 64, tok);
      }
      __syncwarp();
      if (++k == P.nk) k = 0, ++tile;
      if (++s == P.nb) s = 0, parity ^= 1u;
    }
    // every copy has landed before the CTA (and its shared memory) goes
    for (int j = max(0, it - P.nb); j < it; ++j) wait(&bF[j % P.nb], (uint32_t)(j / P.nb) & 1u, true);
  } else if (warp == 2) {
    // ------------------------------------------------------------ codes and grids
    int it = 0, s = 0, k = first_k, tile = tile0;
    uint32_t parity = 1;
    for (; it < count; ++it) {
      if (!wait(&cE[s], parity)) break;
      if (elected()) {
        const int cb = tile / P.token_tiles;
        mbar_expect_tx(&cF[s], CODES + GRIDS * GRID);
        bulk_load(codes + s * CODES, P.codes + ((int64_t)k * P.kblocks + cb) * CODES, CODES, &cF[s]);
#pragma unroll
        for (int j = 0; j < (int)GRIDS; ++j) {
          const int g = P.G == 1 ? 0 : min((cb * 4 + j) / P.chunks, P.G - 1);
          const int64_t at = g * P.mp + (int64_t)k * LIN_BLOCK;
          unsigned char* to = grids + (s * GRIDS + j) * GRID;
          bulk_load(to, P.scales + at, LIN_BLOCK * 4, &cF[s]);
          bulk_load(to + LIN_BLOCK * 4, P.zeros + at, LIN_BLOCK, &cF[s]);
        }
      }
      __syncwarp();
      if (++k == P.nk) k = 0, ++tile;
      if (++s == P.nc) s = 0, parity ^= 1u;
    }
    for (int j = max(0, it - P.nc); j < it; ++j) wait(&cF[j % P.nc], (uint32_t)(j / P.nc) & 1u, true);
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs
    const uint32_t idesc = idesc_f16(128, P.bn) | 1u << 15;
    int sa = 0, sb = 0, k = first_k, more = 0;      // more: blocks in the sum so far
    uint32_t pa = 0, pb = 0, g = 0;
    for (int it = 0; it < count; ++it) {
      if ((!more && !wait(&accE[g & 1u], ((g >> 1) & 1u) ^ 1u)) || !wait(&bF[sb], pb) || !wait(&aF[sa], pa)) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t d = tmem + (g & 1u) * cols;
      const uint64_t a = pair_desc(smem_u32(smem) + sa * FB_A, true), b = smem_desc(smem_u32(tokens) + sb * 2 * half_b);
      const bool last = it == count - 1 || k == P.nk - 1 || more == FB_GROUP - 1;
      if (elected()) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          mma_bf16(d, a + (kk >> 2) * (FB_A / 2 >> 4) + (kk & 3) * (2048 >> 4), b + (kk >> 2) * (half_b >> 4) + (kk & 3) * 2,
                   idesc, more || kk > 0 ? 1u : 0u);
        mma_commit(&aE[sa]);
        mma_commit(&bE[sb]);
        if (last) mma_commit(&accF[g & 1u]);
      }
      __syncwarp();
      more = last ? 0 : more + 1;
      if (last) ++g;
      if (++k == P.nk) k = 0;
      if (++sa == P.na) sa = 0, pa ^= 1u;
      if (++sb == P.nb) sb = 0, pb ^= 1u;
    }
    if (elected()) mma_commit(&done);
    __syncwarp();
    wait(&done, 0, true);
  } else if (warp >= 8) {
    // ------------------------------------------------------------ operands
    // Teams take blocks in turn: what a block costs beside its codes, mostly waits, is hidden by the
    // other teams (16 warps on one block took 16 tokens x 28672 x 8192 8 us more).  A thread takes 32 codes
    // of each of 4 rows: lanes 0-7 eight rows of a unit, the next eight the same rows of the next
    // unit, ..., so that eight lanes' 16-byte loads and stores cover the banks.
    const int t = lane >> 3, r0 = (warp % TEAM) * 8 + (lane & 7);
    const float factor = scale_factor(P.top);
    for (int it = (warp - 8) / TEAM; it < count; it += TEAMS) {
      const int c = it % P.nc, s = it % P.na;
      if (!wait(&cF[c], (uint32_t)(it / P.nc) & 1u)) break;
      if (!wait(&aE[s], ((uint32_t)(it / P.na) & 1u) ^ 1u)) break;
      const unsigned char *here = codes + c * CODES, *grid = grids + c * GRIDS * GRID;
      unsigned char* to = smem + s * FB_A + (r0 & 63) * 128;
#pragma unroll
      for (int i = 0; i < LIN_BLOCK / 8 / TEAM; ++i) {
        const int r = r0 + i * 8 * TEAM;
        uint4 u[W8 ? 2 : 1];
#pragma unroll
        for (int h = 0; h < (W8 ? 2 : 1); ++h) u[h] = *reinterpret_cast<const uint4*>(here + ((4 * h + t) * LIN_BLOCK + r) * 16);
        RowGrid rg[GRIDS];
#pragma unroll
        for (int j = 0; j < (int)GRIDS; ++j)
          rg[j].set(reinterpret_cast<const float*>(grid + j * GRID)[r] * factor, grid[j * GRID + LIN_BLOCK * 4 + r]);
        unsigned char* a = to + (i * 8 * TEAM / 64) * (FB_A / 2) + (i * 8 * TEAM % 64) * 128;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t o[4];
#pragma unroll
          for (int p = 0; p < 4; ++p) o[p] = operand(u, j, p, rg[ONE ? 0 : j]);
          *reinterpret_cast<uint4*>(a + (j >> 1) * 8192 + (((4 * (j & 1) + t) ^ (r & 7)) << 4)) =
              make_uint4(o[0], o[1], o[2], o[3]);
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&cE[c]);
        mbar_arrive(&aF[s]);
      }
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------ sums
    const int q = warp & 3;
    int64_t u = u0;
    pdl_wait();
    for (uint32_t g = 0; u < u1; ++g) {
      const int tile = (int)(u / P.nk);
      const int64_t begin = (int64_t)tile * P.nk, end = begin + P.nk, from = max(begin, u0), to = min(end, u1);
      const int64_t next = min(u + FB_GROUP, to);
      const bool more = u > from, out_now = next == end && from == begin;      // (a whole tile, its last blocks)
      const int tok0 = tile % P.token_tiles * P.bn, tokens = min(P.bn, P.rows - tok0);
      const int col = tile / P.token_tiles * LIN_BLOCK + q * 32 + lane;
      __nv_bfloat16* out = P.dx + (int64_t)tok0 * P.ldx + col;
      if (!wait(&accF[g & 1u], (g >> 1) & 1u)) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      float* mine = P.part + share.slot(blockIdx.x, tile) * P.bn * LIN_BLOCK + q * 32 + lane;
      for (int c = 0; c < tokens; c += 16) {
        uint32_t v[16];
        float sum[16];
        tmem_ld16(tmem + (g & 1u) * cols + ((uint32_t)(q * 32) << 16) + c, v);
        if (more) {      // of the blocks before: loads that wait for no store (rows past the last token are the part's own)
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[i] = mine[(c + i) * LIN_BLOCK];
        }
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] = more ? sum[i] + __uint_as_float(v[i]) : __uint_as_float(v[i]);
        if (!out_now) {
#pragma unroll
          for (int i = 0; i < 16; ++i) mine[(c + i) * LIN_BLOCK] = sum[i];
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (c + i < tokens && col < P.n)
              out[(c + i) * P.ldx] = __float2bfloat16_rn(times(sum[i], P.power[tok0 + c + i]));
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&accE[g & 1u]);
      u = next;
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  pdl_trigger();      // the sum of the parts may get ready; it waits for this grid's end
  if (threadIdx.x == 0) P.flags[blockIdx.x] = abort_flag ? BAKRON_ERR_TIMEOUT : 0;
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * cols) : "memory");
}

// Tiles that several CTAs share: their parts' sum.  A thread has 4 columns of a token.
__global__ void __launch_bounds__(256) k_back_join(const FusedParams P, int ctas) {
  pdl_wait();
  if (blockIdx.x + blockIdx.y == 0) {
    const int bad = __syncthreads_or((int)threadIdx.x < ctas && P.flags[threadIdx.x] != 0);
    if (threadIdx.x == 0) *P.status = bad ? BAKRON_ERR_TIMEOUT : 0;
  }
  const Shares share(P, ctas);
  const int tile = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  const int tok = i >> 5, token = tile % P.token_tiles * P.bn + tok;
  const int col = tile / P.token_tiles * LIN_BLOCK + (i & 31) * 4;
  const int c0 = share.owner((int64_t)tile * P.nk), c1 = share.owner((int64_t)(tile + 1) * P.nk - 1);
  if (c0 == c1 || tok >= P.bn || token >= P.rows || col >= P.n) return;
  const float* from = P.part + (int64_t)tok * LIN_BLOCK + (i & 31) * 4;
  const int64_t size = (int64_t)P.bn * LIN_BLOCK;
  float4 v = *reinterpret_cast<const float4*>(from + share.slot(c0, tile) * size);
#pragma unroll 4
  for (int c = c0 + 1; c <= c1; ++c) {      // (a CTA between the first and the last has nothing else)
    const float4 w = *reinterpret_cast<const float4*>(from + (int64_t)c * 2 * size);
    v.x += w.x;
    v.y += w.y;
    v.z += w.z;
    v.w += w.w;
  }
  const float2 power = P.power[token];
  v = make_float4(times(v.x, power), times(v.y, power), times(v.z, power), times(v.w, power));
  __nv_bfloat16* out = P.dx + token * P.ldx + col;
  if (P.vec && col + 4 <= P.n) {
    *reinterpret_cast<uint2*>(out) = make_uint2(bf16_pack(v.x, v.y), bf16_pack(v.z, v.w));
  } else {
    const float o[4] = {v.x, v.y, v.z, v.w};
    for (int k = 0; k < 4 && col + k < P.n; ++k) out[k] = __float2bfloat16_rn(o[k]);
  }
}

// ------------------------------------------------------------------ many tokens

struct ExpandParams {
  const unsigned char* codes;
  const float* scales;
  const uint8_t* zeros;
  int m, kblocks, chunks, G;
  int64_t mp;
  const int* top;
  __half* w;
  int64_t ldw;      // a multiple of 128
};

// What in fp16, row by row.  A thread takes a 16-byte unit; four lanes have a row's chunk together.  11008 x 4096: 20 us.
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
  const float factor = scale_factor(P.top);
#pragma unroll
  for (int j = 0; j < (W8 ? 2 : 4); ++j) {
    const int chunk = kb * 4 + (W8 ? half * 2 : 0) + j, grid = P.G == 1 ? 0 : min(chunk / P.chunks, P.G - 1);
    RowGrid g;
    g.set(P.scales[grid * P.mp + row] * factor, P.zeros[grid * P.mp + row]);
    uint32_t o[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) o[p] = W8 ? operand8(words[2 * j + (p >> 1)], p & 1, g) : operand4(words[j], p, g);
    *reinterpret_cast<uint4*>(P.w + row * P.ldw + chunk * 32 + 8 * t) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

constexpr int FUSED_TOKENS = 2048;               // at most by the fused kernel
constexpr uint32_t FB_SMEM = 227 * 1024 - 1024;      // beside the barriers

bool one_grid(int n, int group_size) { return group_size == 0 || group_size == n || group_size % LIN_BLOCK == 0; }

// How the fused kernel's tokens are shared out.
static_assert(ROW_SMS <= 256, "a thread a flag");
struct FusedPlan {
  int bn, token_tiles, tiles, nk, ctas, teams, na, nb, nc;
  size_t smem;
  FusedPlan(int rows, int m, int n, bool bytes8, bool one) {
    bn = (int)round_up(ceil_div(rows, ceil_div(rows, FB_MAX_BN)), 16);      // as even as tiles allow
    token_tiles = ceil_div(rows, bn);
    tiles = ceil_div(n, LIN_BLOCK) * token_tiles;
    nk = ceil_div(m, LIN_BLOCK);
    // every SM, but no fewer than 4 blocks each: a part costs its sums' way through memory
    ctas = (int)std::max<int64_t>(1, std::min<int64_t>(ROW_SMS, (int64_t)tiles * nk / 4));
    const uint32_t tok = (uint32_t)bn * 256, code = (bytes8 ? 16384 : 8192) + LIN_BLOCK * 5 * (one ? 1 : 4);
    auto fits = [&](int a, int b, int c) { return 1024 + a * FB_A + b * tok + c * code <= FB_SMEM; };
    na = teams = fits(4, 2, 4) ? 4 : 2;      // (two blocks of operands always fit)
    nb = 2;
    nc = fits(na, nb, 4) ? 4 : 2;
    while (nb < FB_RING && fits(na, nb + 1, nc)) ++nb;
    smem = 1024 + na * FB_A + nb * tok + nc * code;
  }
};

// Which way more than 8 tokens go: estimates of both in us, fitted to 12 shapes of m and n from 512 to 28672 (4 and 8
// bits) at 64 to 2048 tokens, where the rule's choice is at most 7% behind the other.  Fused: blocks a CTA, sums of whole tiles
// that leave after the last block or slower than the next tile's blocks go by, the parts of shared tiles.  Else: rounds of the
// pairs, the weight written out.  512 tokens: 4096 x 4096 40 fused, 42 else, 11008 x 4096 70 and 84, 28672 x 512 41 and 150,
// 4096 x 11008 84 and 74, 28672 x 8192 280 and 244; 1024: 74, 45; 131, 92; 69, 160; 141, 94; 536, 382.
bool fused_is_faster(const FusedPlan& F, int rows, int m, int n, bool bytes8) {
  if (rows > FUSED_TOKENS) return false;
  const double per = (double)F.tiles / F.ctas, blocks = per * F.nk, bn = F.bn, million = 1e-6;
  double fused = 13.6 + blocks * (0.47 + 0.0026 * bn) + 0.75 * million * rows * m;
  if (F.tiles >= F.ctas)
    fused += 0.096 * bn + 1.1 * per * std::max(0., 0.09 * bn - F.nk * (0.6 + 0.0018 * bn));
  else
    fused += 3.7 * million * rows * n;
  const int rounds = ceil_div(ceil_div(rows, PG_M) * ceil_div(n, 256), PG_PAIRS);
  const double written = 15.6 + 0.27 * rounds * ceil_div(m, PG_K) + (bytes8 ? 0.70 : 0.43) * million * m * n +
                         million * rows * (0.76 * m + 0.30 * n);
  return fused <= written;
}

// How up to 8 tokens are: the rows in so many parts (64 at most) that the CTAs, as many at a time as the SMs hold, are done
// first, where a CTA costs 256 rows (16 chunks) beside its own.  1 token x 28672 x 8192, 64 tiles: 4 parts (256 CTAs of 304)
// 59 us, 9 (576 of 608) 55, 14 56; 4096 x 11008, 86 tiles: 3 parts 18, 4 20.
struct FewPlan {
  int tiles, chunks, per, splits;
  FewPlan(int m, int n, bool bytes8, bool one) {
    tiles = ceil_div(n, FW_COLS);
    chunks = ceil_div(m, 16);
    const int slots = few_ctas(bytes8, one) * ROW_SMS;
    int64_t best = INT64_MAX;
    for (int s = 1; s <= 64; ++s) {
      const int rows = (int)round_up(ceil_div(chunks, s), FW_WARPS), parts = ceil_div(chunks, rows);
      const int64_t cost = (int64_t)ceil_div(tiles * parts, slots) * (rows + 16);
      if (cost >= best) continue;
      best = cost;
      per = rows;
      splits = parts;
    }
  }
};

struct BackLayout {
  size_t dy = 0, power = 0, flags = 0, part = 0, w = 0, bytes;
  int64_t ldy, ldw;      // of the gradients, of the weight, both in fp16
  bool fused;
  BackLayout(int rows, int m, int n, bool bytes8, bool one, const FusedPlan& F) {
    size_t at = 256;
    auto take = [&](size_t b) {
      const size_t r = at;
      at += align256(b);
      return r;
    };
    fused = fused_is_faster(F, rows, m, n, bytes8);
    ldy = round_up(m, 8);
    ldw = round_up(n, LIN_BLOCK);
    if (rows > FEW_BACK) {
      dy = take((size_t)rows * ldy * 2);
      power = take((size_t)rows * sizeof(float2));
    }
    if (rows <= FEW_BACK) {
      const FewPlan few(m, n, bytes8, one);
      part = take((size_t)few.splits * rows * few.tiles * FW_COLS * 4);
    } else if (fused) {
      flags = take((size_t)F.ctas * sizeof(int));
      part = take((size_t)F.ctas * 2 * F.bn * LIN_BLOCK * 4);
    } else {
      w = take((size_t)m * ldw * 2);
    }
    bytes = at;
  }
};

template <bool W8, bool ONE>
cudaError_t few_launch(const FewParams& P, const FewPlan& F, cudaStream_t s) {
  const dim3 grid((unsigned)F.tiles, (unsigned)F.splits);
  const auto kernel = P.rows <= 4 ? (P.yvec ? k_back_few<W8, ONE, true, true> : k_back_few<W8, ONE, true, false>)
                                  : (P.yvec ? k_back_few<W8, ONE, false, true> : k_back_few<W8, ONE, false, false>);
  kernel<<<grid, FW_WARPS * 32, FW_SMEM, s>>>(P);
  return cudaGetLastError();
}

template <bool W8, bool ONE, int TEAMS>
cudaError_t fused_launch(const CUtensorMap& map, const FusedParams& P, const FusedPlan& F, cudaStream_t s) {
  static OncePerDevice once;
  const cudaError_t e = once([] {
    return cudaFuncSetAttribute(k_back_fused<W8, ONE, TEAMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)FB_SMEM);
  });
  if (e != cudaSuccess) return e;
  return launch_pdl(k_back_fused<W8, ONE, TEAMS>, dim3((unsigned)F.ctas), dim3(FB_THREADS), F.smem, s, map, P);
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
  return back_ok(rows, m, n, qmax, group_size) && rows > 0
             ? BackLayout(rows, m, n, qmax > 15, one_grid(n, group_size), FusedPlan(rows, m, n, qmax > 15, one_grid(n, group_size))).bytes
             : 0;
}

extern "C" int bakron_linear_backward(const void* dy, int rows, int64_t lddy, const void* packed, int m, int n, int qmax,
                                      int group_size, void* dx, int64_t lddx, void* workspace, size_t workspace_bytes,
                                      int sync, void* stream) {
  if (!back_ok(rows, m, n, qmax, group_size)) return BAKRON_ERR_INVALID_ARG;
  if (rows == 0) return BAKRON_OK;
  if (!dy || !packed || !dx || lddy < m || lddx < n || (uintptr_t)packed % 16 != 0 || (uintptr_t)dy % 2 != 0 ||
      (uintptr_t)dx % 2 != 0 || !workspace || (uintptr_t)workspace % 16 != 0)
    return BAKRON_ERR_INVALID_ARG;
  const bool one = one_grid(n, group_size);
  const FusedPlan plan(rows, m, n, qmax > 15, one);
  const BackLayout B(rows, m, n, qmax > 15, one, plan);
  if (workspace_bytes < B.bytes) return BAKRON_ERR_WORKSPACE;
  const WeightLayout L(m, n, qmax, group_size);
  const unsigned char* p = (const unsigned char*)packed;
  cudaStream_t s = (cudaStream_t)stream;
  char* ws = (char*)workspace;
  if (rows <= FEW_BACK) {
    const FewPlan few(m, n, L.bytes8, one);
    FewParams F{p + L.off_codes, (const float*)(p + L.off_scales), p + L.off_zeros, L.mp, (int)(L.np / LIN_BLOCK),
                L.G == 1 ? (int)(L.np / 32) : L.group / 32, (int)L.G, rows, m, n, few.chunks, few.per,
                (const __nv_bfloat16*)dy, lddy, m % 4 == 0 && ((uintptr_t)dy | (uintptr_t)(rows > 1 ? lddy * 2 : 0)) % 8 == 0,
                (float*)(ws + B.part), (int*)ws};
    const auto launch = L.bytes8 ? (one ? few_launch<true, true> : few_launch<true, false>)
                                 : (one ? few_launch<false, true> : few_launch<false, false>);
    BK_CUDA_OK(launch(F, few, s));
    BK_CUDA_OK(launch_pdl(k_back_few_sum, dim3((unsigned)ceil_div(n, 256), (unsigned)rows), dim3(256), 0, s, F.part, few.splits,
                          rows, few.tiles, n, (__nv_bfloat16*)dx, lddx));
    return sync ? bakron_read_status(workspace, stream) : BAKRON_OK;
  }
  const int* top = (const int*)p + 1;
  float2* power = (float2*)(ws + B.power);
  const auto tokens = aligned16(dy, rows > 1 ? lddy * 2 : 0) ? k_back_tokens<true> : k_back_tokens<false>;
  tokens<<<(unsigned)rows, 512, 0, s>>>((const __nv_bfloat16*)dy, lddy, m, top, (__half*)(ws + B.dy), B.ldy, power,
                                        B.fused ? nullptr : (int*)ws);
  BK_CUDA_OK(cudaGetLastError());
  dy = ws + B.dy;
  CUtensorMap a, b, o;
  if (B.fused) {
    if (!pair_map(&a, false, dy, rows, m, B.ldy, 64, plan.bn)) return BAKRON_ERR_CUDA;
    FusedParams F{p + L.off_codes, (const float*)(p + L.off_scales), p + L.off_zeros, L.mp, (int)(L.np / LIN_BLOCK),
                  L.G == 1 ? (int)(L.np / 32) : L.group / 32, (int)L.G, rows, n, plan.bn, plan.nk, plan.token_tiles,
                  plan.tiles, plan.na, plan.nb, plan.nc, top, power, (__nv_bfloat16*)dx, lddx, (float*)(ws + B.part),
                  aligned16(dx, rows > 1 ? lddx * 2 : 0), (int*)ws, (int*)(ws + B.flags),
                  spin_cycles_from_env()};
    const auto launch =
        plan.teams == 4 ? (L.bytes8 ? (one ? fused_launch<true, true, 4> : fused_launch<true, false, 4>)
                                    : (one ? fused_launch<false, true, 4> : fused_launch<false, false, 4>))
                        : (L.bytes8 ? (one ? fused_launch<true, true, 2> : fused_launch<true, false, 2>)
                                    : (one ? fused_launch<false, true, 2> : fused_launch<false, false, 2>));
    BK_CUDA_OK(launch(a, F, plan, s));
    BK_CUDA_OK(launch_pdl(k_back_join, dim3((unsigned)ceil_div(plan.bn, 8), (unsigned)plan.tiles), dim3(256), 0, s, F,
                            plan.ctas));
    return sync ? bakron_read_status(workspace, stream) : BAKRON_OK;
  }
  ExpandParams E{p + L.off_codes, (const float*)(p + L.off_scales), p + L.off_zeros, m, (int)(L.np / LIN_BLOCK),
                 L.G == 1 ? (int)(L.np / 32) : L.group / 32, (int)L.G, L.mp, top, (__half*)(ws + B.w), B.ldw};
  const unsigned ctas = (unsigned)(L.mp * E.kblocks * (L.units / 4) / 64);
  L.bytes8 ? k_expand<true><<<ctas, 256, 0, s>>>(E) : k_expand<false><<<ctas, 256, 0, s>>>(E);
  BK_CUDA_OK(cudaGetLastError());
  PairShape S{};
  S.tm = ceil_div(rows, PG_M);
  S.tn = ceil_div(n, 256);
  S.bn = 256;
  S.nk = S.per = ceil_div(m, PG_K);
  S.group = PG_GROUP;
  S.splits = 1;
  S.band = 16;
  S.half = 1;
  S.rows = rows;
  S.a_rows = 128;
  S.status = (int*)ws;
  S.spin_cycles = spin_cycles_from_env();
  const bool tma = aligned16(dx, rows > 1 ? lddx * 2 : 0);
  if (!pair_map(&a, false, dy, rows, m, B.ldy, PG_K, S.a_rows) ||
      !pair_map(&b, false, E.w, m, n, B.ldw, 64, PG_K) ||
      (tma && !pair_map(&o, false, dx, rows, n, rows > 1 ? lddx : round_up(n, 8), 64, 32)))
    return BAKRON_ERR_CUDA;
  EpiBf16::Params T{tma ? nullptr : (__nv_bfloat16*)dx, lddx, rows, n, nullptr, nullptr, 0, power};
  BK_CUDA_OK((pair_launch<EpiBf16, false, true>(a, b, tma ? o : a, S, T, s)));
  return sync ? bakron_read_status(workspace, stream) : BAKRON_OK;
}
