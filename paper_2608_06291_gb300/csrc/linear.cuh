// The weight of bakron_linear as bakron_pack_weight lays it out, and the kernels'
// common parameters.
//
// [status 256 B][scales G x mp fp32][zeros G x mp uint8][codes]
//
// mp: m rounded up to 128, np: n rounded up to 128, G: grids a row.  Codes lie in blocks
// of 128 rows x 128 columns, [row block][column block][unit][row] of 16-byte units, so
// that a row's unit is next to its neighbours' (a warp reads whole 128-byte lines) and a
// block is one contiguous copy.  With 4 bits a code (qmax <= 15) a block has 4 units a
// row; word j (0..3) of unit t holds the 8 columns 32 j + 8 t + (0..7), so a unit has a
// piece of each 32-column chunk (a chunk has one grid), and a warp's four lanes of a
// row read a chunk's columns in order.  With 8 bits it has 8 units; unit t + 4 h holds those
// columns of the chunks 2 h and 2 h + 1, two words each.  Inside a word, columns are
// ordered so that the two of a pair come out in the two halves of a register:
//   4 bits  columns 0..7 at nibbles 0 4 1 5 2 6 3 7
//   8 bits  columns 0..3 at bytes 0 2 1 3
// Padding rows have scale 0, padding columns the code that stands for 0.
#pragma once

#include "rowops.cuh"

namespace bakron {

constexpr int LIN_BLOCK = 128;

struct WeightLayout {
  int64_t mp, np, G;
  int group;          // columns a grid covers (n for one grid a row)
  bool bytes8;        // 8 bits a code
  int units;          // 16-byte units of a row's block
  size_t off_scales, off_zeros, off_codes, bytes;
  WeightLayout(int m, int n, int qmax, int group_size) {
    mp = round_up(m, LIN_BLOCK);
    np = round_up(n, LIN_BLOCK);
    G = group_size ? n / group_size : 1;
    group = group_size ? group_size : n;
    bytes8 = qmax > 15;
    units = bytes8 ? 8 : 4;
    off_scales = 256;
    off_zeros = align256(off_scales + size_t(G * mp) * 4);
    off_codes = align256(off_zeros + size_t(G * mp));
    bytes = off_codes + size_t(mp * (np / LIN_BLOCK)) * units * 16;
  }
};

struct LinearParams {
  const void* x;
  int64_t ldx;
  const float* xscales;     // a scale per token, or null
  const unsigned char* codes;
  const float* scales;
  const uint8_t* zeros;
  const float* bias;
  const void* residual;     // y's type
  int64_t ldr;
  void* y;
  int64_t ldy;
  int rows, m, n;
  int64_t mp;
  int kblocks;              // 128-column blocks
  int chunks;               // 32-column chunks of a grid
  int G;
  int activation, yf32;
  int xvec;                 // x can be read 8 elements at a time
  int yvec;                 // y and the residual 16 bytes at a time, from columns that are multiples of 8
  int* status;              // the call's status word, or null
};

// erf to 1.5e-7 (Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26), for bf16
// results: erff cost the epilogue of a 4096 x 28672 product 100 us, erfcf in an fp32 one 150 (846 -> 996).
__device__ __forceinline__ float erf_short(float v) {
  const float x = fabsf(v), t = __fdividef(1.f, fmaf(0.3275911f, x, 1.f));
  float p = fmaf(1.061405429f, t, -1.453152027f);
  p = fmaf(p, t, 1.421413741f);
  p = fmaf(p, t, -0.284496736f);
  p = fmaf(p, t, 0.254829592f) * t;
  return copysignf(fmaf(-p, __expf(-x * x), 1.f), v);
}

// EXACT: for fp32 results, right but for a few of their last bits (erfc, as 1 + erf cancels where
// v is negative).  Else for results that are rounded to bf16: what the short forms lose is far
// below its 2^-9, but for GELU's tail (below -4, where it errs by up to 1e-7 |v|).
template <bool EXACT>
__device__ __forceinline__ float activate(float v, int a) {
  switch (a) {
    case BAKRON_RELU: return v < 0.f ? 0.f : v;     // NaN stays
    case BAKRON_SILU:      // the divisor's overflow gives 0, as it should
      return EXACT ? v / (1.f + expf(-v)) : __fdividef(v, 1.f + __expf(-v));
    case BAKRON_GELU:
      return EXACT ? 0.5f * v * erfcf(v * -0.70710678f) : 0.5f * v * (1.f + erf_short(v * 0.70710678f));
    default: return v;
  }
}
__host__ __device__ __forceinline__ bool exact_activation(const LinearParams& P) {
  return P.yf32 && P.activation >= BAKRON_SILU;
}

// One entry from the product's sum to its store.
template <bool EXACT>
__device__ __forceinline__ void linear_store(const LinearParams& P, float v, int64_t tok, int row) {
  if (P.xscales) v *= P.xscales[tok];
  if (P.bias) v += P.bias[row];
  v = activate<EXACT>(v, P.activation);
  if (P.residual)
    v += P.yf32 ? ((const float*)P.residual)[tok * P.ldr + row]
                : __bfloat162float(((const __nv_bfloat16*)P.residual)[tok * P.ldr + row]);
  if (P.yf32)
    ((float*)P.y)[tok * P.ldy + row] = v;
  else
    ((__nv_bfloat16*)P.y)[tok * P.ldy + row] = __float2bfloat16_rn(v);
}
__device__ __forceinline__ void linear_store(const LinearParams& P, float v, int64_t tok, int row) {
  exact_activation(P) ? linear_store<true>(P, v, tok, row) : linear_store<false>(P, v, tok, row);
}

// Two codes of a pair as bf16 values c - z, exact: integers up to 255.
// 4 bits: 0x4300 | c is 128 + c; z128 holds 128 + z twice.
__device__ __forceinline__ uint32_t pair4(uint32_t word, int p, __nv_bfloat162 z128) {
  uint32_t v = ((word >> (4 * p)) & 0x000F000Fu) | 0x43004300u;
  __nv_bfloat162 r = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&v), z128);
  return *reinterpret_cast<uint32_t*>(&r);
}
// 8 bits: c = 16 h + l; ((h 16 - z) + l), every step an integer of at most 8 bits.
__device__ __forceinline__ uint32_t pair8(uint32_t w0, uint32_t w1, int p, __nv_bfloat162 z) {
  const uint32_t v = (p < 2 ? w0 : w1) >> (8 * (p & 1));
  uint32_t l = (v & 0x000F000Fu) | 0x43004300u, h = ((v >> 4) & 0x000F000Fu) | 0x43004300u;
  const __nv_bfloat162 k = __float2bfloat162_rn(128.f), c16 = __float2bfloat162_rn(16.f);
  const __nv_bfloat162 hh = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&h), k);
  const __nv_bfloat162 ll = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&l), k);
  __nv_bfloat162 r = __hadd2(__hfma2(hh, c16, __hneg2(z)), ll);
  return *reinterpret_cast<uint32_t*>(&r);
}

// Many tokens (linear_tc.cu): the bytes of workspace its call needs (the status, the tokens'
// copy where they cannot be read as they are), and the call.
size_t linear_tc_workspace(const void* x, bool x8, int rows, int64_t ldx, int n, bool bytes8);
int linear_tc(const LinearParams& L, bool x8, bool bytes8, void* workspace, cudaStream_t s);

}  // namespace bakron
