// bakron_pack_weight and bakron_linear: y = act(x What^T + b) + r on a quantised weight,
// What_ij = s (c_ij - z) with the grid (s, z) of row i and j's group.
//
// c - z is an integer of at most 8 bits, so it is exact as an operand of the tensor cores
// and so are its products with bf16 (or e4m3) values in fp32; the scale of a group
// multiplies the group's fp32 sum.
#include "linear.cuh"

namespace bakron {
namespace {

// ------------------------------------------------------------------ layout
struct PackParams {
  const uint8_t* codes;
  int64_t ldc;
  const float *scales, *zeros;
  int m, n, qmax, group;
  int64_t mp, G;
  int kblocks, units;
  float* pscales;
  uint8_t* pzeros;
  unsigned char* pcodes;
  int* status;
};

__device__ __forceinline__ float grid_zero(const PackParams& P, int row, int64_t g) {
  return P.zeros[row * P.G + g];
}

__global__ void __launch_bounds__(256) k_pack_grid(const PackParams P) {
  const int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
  const int64_t g = i / P.mp;
  const int row = (int)(i % P.mp);
  const bool there = i < P.G * P.mp;
  float s = 0.f, z = 0.f;
  if (there && row < P.m) {
    s = P.scales[row * P.G + g];
    z = grid_zero(P, row, g);
    if (!(z >= 0.f && z <= (float)P.qmax && z == floorf(z))) {
      raise_status(P.status, BAKRON_ERR_INVALID_ARG);
      z = 0.f;
    }
  }
  if (there) {
    P.pscales[i] = s;
    P.pzeros[i] = (uint8_t)z;
  }
  // one atomic a CTA, of a maximum: in any order the same
  __shared__ int most[8];
  int e = (int)(__float_as_uint(s) >> 23) & 255;
  e = (int)__reduce_max_sync(0xffffffffu, (unsigned)(e == 255 ? 0 : e));
  if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = e;
  __syncthreads();
  if (threadIdx.x > 0) return;
  for (int w = 1; w < 8; ++w) e = max(e, most[w]);
  if (e > 0) atomicMax(P.status + 1, e);
}

// One 16-byte unit per thread.
__global__ void __launch_bounds__(256) k_pack_codes(const PackParams P) {
  const int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
  if (i >= P.mp * P.kblocks * P.units) return;
  const int in = (int)(i % LIN_BLOCK);
  const int64_t rest = i / LIN_BLOCK;
  const int unit = (int)(rest % P.units), kb = (int)(rest / P.units % P.kblocks);
  const int64_t row = rest / P.units / P.kblocks * LIN_BLOCK + in;
  auto code = [&](int col) -> uint32_t {
    if (row >= P.m) return 0u;
    if (col >= P.n) {
      const float z = grid_zero(P, (int)row, P.G - 1);
      return z >= 0.f && z <= (float)P.qmax ? (uint32_t)z : 0u;
    }
    const uint32_t c = P.codes[row * P.ldc + col];
    if (c > (uint32_t)P.qmax) {
      raise_status(P.status, BAKRON_ERR_INVALID_ARG);
      return 0u;
    }
    return c;
  };
  uint32_t w[4];
  if (P.units == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c0 = kb * LIN_BLOCK + 32 * j + 8 * unit;
      w[j] = 0u;
#pragma unroll
      for (int e = 0; e < 8; ++e) w[j] |= code(c0 + e) << (4 * (e / 2 + 4 * (e % 2)));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c0 = kb * LIN_BLOCK + 32 * (2 * (unit >> 2) + j / 2) + 8 * (unit & 3) + 4 * (j % 2);
      w[j] = 0u;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[j] |= code(c0 + e) << (8 * (e / 2 + 2 * (e % 2)));
    }
  }
  reinterpret_cast<uint4*>(P.pcodes)[i] = make_uint4(w[0], w[1], w[2], w[3]);
}

// ------------------------------------------------------------------ few tokens
// D (16 x 8) += A (16 x 16, bf16) B (16 x 8, bf16), fp32 accumulators.
__device__ __forceinline__ void mma_bf16_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                                 uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 8 elements of a token as bf16 pairs, zeros past n and past the last token.
template <bool X8>
__device__ __forceinline__ void load_x8(const LinearParams& P, int64_t tok, int k, uint32_t (&b)[4]) {
  b[0] = b[1] = b[2] = b[3] = 0u;
  if (tok >= P.rows || k >= P.n) return;
  if constexpr (X8) {
    const uint8_t* p = (const uint8_t*)P.x + tok * P.ldx + k;
    uint2 q = make_uint2(0u, 0u);
    if (P.xvec && k + 8 <= P.n) {
      q = *reinterpret_cast<const uint2*>(p);
    } else {
      uint8_t* e = reinterpret_cast<uint8_t*>(&q);
      for (int j = 0; j < 8 && k + j < P.n; ++j) e[j] = p[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t two = (j < 2 ? q.x : q.y) >> (16 * (j & 1));
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xFFFFu), __NV_E4M3);
      const float2 f = __half22float2(__half2(h));
      b[j] = bf16_pack(f.x, f.y);    // exact: e4m3 has 4 significant bits
    }
  } else {
    const __nv_bfloat16* p = (const __nv_bfloat16*)P.x + tok * P.ldx + k;
    if (P.xvec && k + 8 <= P.n) {
      const uint4 q = *reinterpret_cast<const uint4*>(p);
      b[0] = q.x; b[1] = q.y; b[2] = q.z; b[3] = q.w;
    } else {
      const uint16_t* e = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k + j < P.n) b[j / 2] |= (uint32_t)e[j] << (16 * (j & 1));
    }
  }
}

constexpr int FEW_ROWS = 32;     // rows of What a CTA takes
constexpr int FEW_WARPS = 8;     // they share its columns, block by block

// 32 rows x 8 NT tokens per CTA.  What's rows are the rows of mma.sync's first operand,
// read straight from the packed units into its registers; the tokens are its columns.
// Bound by its waits, not by memory (1 token x 8192 x 8192 in groups of 128: 28 us, DRAM 16% busy,
// issue 34%): a new grid's scales and zeros and a block's tokens are loaded where they are
// used, and codes are only one block ahead.  As graph replays: 1 x 28672 x 8192, 118 MB of codes, 58 us
// in groups of 128 (2.2 TB/s with the grids), 41 with one grid a row; 1 x 4096 x 4096 10.  CTAs
// an SM as registers allow (two of 16 tokens x 8-bit codes spill: 29 us for 4099 x 11008, one 25).
template <int NT, bool W8, bool X8>
__global__ void __launch_bounds__(FEW_WARPS * 32, W8 ? 3 - NT : 4 - NT) k_linear_few(const LinearParams P) {
  constexpr int UW = W8 ? 2 : 1;     // units of a row a lane reads per block
  __shared__ float red[FEW_WARPS][8 * NT][FEW_ROWS + 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int64_t row0 = (int64_t)blockIdx.x * FEW_ROWS, tok0 = (int64_t)blockIdx.y * 8 * NT;
  if (P.status && blockIdx.x + blockIdx.y + threadIdx.x == 0) *P.status = 0;      // nothing here can run out
  const unsigned char* base = P.codes + (row0 / LIN_BLOCK) * P.kblocks * (4 * UW) * 2048 +
                              (row0 % LIN_BLOCK + g) * 16 + t * 2048;
  float acc[2][NT][4] = {}, cur[2][NT][4] = {};
  float s[2][2];
  __nv_bfloat162 z[2][2];
  int grid = -1;
  auto promote = [&]() {
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[mt][n][e] = fmaf(s[mt][e >> 1], cur[mt][n][e], acc[mt][n][e]);
          cur[mt][n][e] = 0.f;
        }
  };
  // the next block's codes are on their way while this one is multiplied (the tokens too took
  // so many registers that 16 tokens x 28672 x 8192 went from 86 to 156 us)
  struct Block {
    uint4 u[2][2][UW];
  };
  auto load = [&](int kb, Block& to) {
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int h = 0; h < UW; ++h)
          to.u[mt][r][h] = __ldg(reinterpret_cast<const uint4*>(
              base + ((int64_t)kb * 4 * UW + 4 * h) * 2048 + (mt * 16 + r * 8) * 16));
  };
  Block next;
  if (warp < P.kblocks) load(warp, next);
  for (int kb = warp; kb < P.kblocks; kb += FEW_WARPS) {
    const Block here = next;
    const auto& u = here.u;
    uint32_t b[NT][4][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        load_x8<X8>(P, tok0 + n * 8 + g, kb * LIN_BLOCK + 32 * j + 8 * t, b[n][j]);
    if (kb + FEW_WARPS < P.kblocks) load(kb + FEW_WARPS, next);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int now = P.G == 1 ? 0 : min((kb * 4 + j) / P.chunks, P.G - 1);
      if (now != grid) {
        if (grid >= 0) promote();
        grid = now;
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int64_t at = grid * P.mp + row0 + mt * 16 + r * 8 + g;
            s[mt][r] = P.scales[at];
            z[mt][r] = __float2bfloat162_rn((float)P.zeros[at] + (W8 ? 0.f : 128.f));
          }
      }
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        uint32_t a[2][4];      // row g, g + 8; pairs of the 8 columns
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            if constexpr (W8) {
              const uint32_t* w = reinterpret_cast<const uint32_t*>(&u[mt][r][j >> 1]);
              a[r][p] = pair8(w[2 * (j & 1)], w[2 * (j & 1) + 1], p, z[mt][r]);
            } else {
              a[r][p] = pair4(reinterpret_cast<const uint32_t*>(&u[mt][r][0])[j], p, z[mt][r]);
            }
          }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            mma_bf16_16x8x16(cur[mt][n], a[0][2 * i], a[1][2 * i], a[0][2 * i + 1], a[1][2 * i + 1],
                             b[n][j][2 * i], b[n][j][2 * i + 1]);
      }
    }
  }
  if (grid >= 0) promote();
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        red[warp][n * 8 + 2 * t + (e & 1)][mt * 16 + (e >> 1) * 8 + g] = acc[mt][n][e];
  __syncthreads();
  for (int i = threadIdx.x; i < FEW_ROWS * 8 * NT; i += FEW_WARPS * 32) {
    const int r = i % FEW_ROWS, c = i / FEW_ROWS;
    if (row0 + r >= P.m || tok0 + c >= P.rows) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < FEW_WARPS; ++w) v += red[w][c][r];
    linear_store(P, v, tok0 + c, (int)(row0 + r));
  }
}

template <int NT>
void launch_few(const LinearParams& P, bool w8, bool x8, cudaStream_t s) {
  const dim3 grid((unsigned)ceil_div(P.m, FEW_ROWS), (unsigned)ceil_div(P.rows, 8 * NT));
  if (w8)
    x8 ? k_linear_few<NT, true, true><<<grid, FEW_WARPS * 32, 0, s>>>(P)
       : k_linear_few<NT, true, false><<<grid, FEW_WARPS * 32, 0, s>>>(P);
  else
    x8 ? k_linear_few<NT, false, true><<<grid, FEW_WARPS * 32, 0, s>>>(P)
       : k_linear_few<NT, false, false><<<grid, FEW_WARPS * 32, 0, s>>>(P);
}

constexpr int LIN_MAX_DIM = 1 << 17, LIN_MAX_ROWS = 1 << 30;
// Up to here the codes' reading is all there is, and mma.sync is enough (16 tokens x 11008 x 4096:
// 19 us, by the tensor-memory kernel 25).
constexpr int FEW_TOKENS = 16;

bool weight_ok(int m, int n, int qmax, int group_size) {
  return m >= 1 && n >= 1 && m <= LIN_MAX_DIM && n <= LIN_MAX_DIM && qmax >= 1 && qmax <= 255 &&
         (group_size == 0 || (group_size > 0 && group_size % 32 == 0 && n % group_size == 0));
}

}  // namespace
}  // namespace bakron

using namespace bakron;

extern "C" size_t bakron_packed_bytes(int m, int n, int qmax, int group_size) {
  return weight_ok(m, n, qmax, group_size) ? WeightLayout(m, n, qmax, group_size).bytes : 0;
}

extern "C" int bakron_pack_weight(const uint8_t* codes, int64_t ldc, const float* scales,
                                  const float* zeros, int m, int n, int qmax, int group_size,
                                  void* packed, size_t packed_bytes, void* stream) {
  if (!codes || !scales || !zeros || !packed || !weight_ok(m, n, qmax, group_size) || ldc < n ||
      (uintptr_t)packed % 16 != 0)
    return BAKRON_ERR_INVALID_ARG;
  const WeightLayout L(m, n, qmax, group_size);
  if (packed_bytes < L.bytes) return BAKRON_ERR_WORKSPACE;
  cudaStream_t s = (cudaStream_t)stream;
  char* p = (char*)packed;
  BK_CUDA_OK(cudaMemsetAsync(p, 0, 256, s));
  PackParams P{codes, ldc, scales, zeros, m, n, qmax, L.group, L.mp, L.G, (int)(L.np / LIN_BLOCK), L.units,
               (float*)(p + L.off_scales), (uint8_t*)(p + L.off_zeros),
               (unsigned char*)(p + L.off_codes), (int*)p};
  const int64_t units = L.mp * (L.np / LIN_BLOCK) * L.units;
  k_pack_grid<<<(unsigned)((L.G * L.mp + 255) / 256), 256, 0, s>>>(P);
  k_pack_codes<<<(unsigned)((units + 255) / 256), 256, 0, s>>>(P);
  BK_CUDA_OK(cudaGetLastError());
  return bakron_read_status(packed, stream);
}

extern "C" size_t bakron_linear_workspace_bytes(const void* x, int xdtype, int rows, int64_t ldx,
                                                int n, int qmax, int group_size) {
  if (rows <= FEW_TOKENS || !weight_ok(1, n, qmax, group_size)) return 0;
  return linear_tc_workspace(x, xdtype == BAKRON_E4M3, rows, ldx, n, qmax > 15);
}

extern "C" int bakron_linear(const void* x, int xdtype, int rows, int64_t ldx, const float* xscales,
                             const void* packed, int m, int n, int qmax, int group_size,
                             const float* bias, int activation, const void* residual, int64_t ldr,
                             void* y, int ydtype, int64_t ldy, void* workspace,
                             size_t workspace_bytes, int sync, void* stream) {
  if (rows < 0 || rows > LIN_MAX_ROWS || !weight_ok(m, n, qmax, group_size) || (xdtype != BAKRON_BF16 && xdtype != BAKRON_E4M3) ||
      (ydtype != BAKRON_BF16 && ydtype != BAKRON_F32) || activation < BAKRON_NO_ACTIVATION ||
      activation > BAKRON_GELU)
    return BAKRON_ERR_INVALID_ARG;
  if (rows == 0) return BAKRON_OK;
  if (!x || !packed || !y || ldx < n || ldy < m || (residual && ldr < m) || (uintptr_t)packed % 16 != 0)
    return BAKRON_ERR_INVALID_ARG;
  const size_t need = bakron_linear_workspace_bytes(x, xdtype, rows, ldx, n, qmax, group_size);
  if (need && (!workspace || (uintptr_t)workspace % 16 != 0)) return BAKRON_ERR_INVALID_ARG;
  if (workspace_bytes < need) return BAKRON_ERR_WORKSPACE;
  const WeightLayout L(m, n, qmax, group_size);
  const unsigned char* p = (const unsigned char*)packed;
  const bool x8 = xdtype == BAKRON_E4M3;
  LinearParams P{};
  P.x = x; P.ldx = ldx; P.xscales = xscales;
  P.codes = p + L.off_codes; P.scales = (const float*)(p + L.off_scales); P.zeros = p + L.off_zeros;
  P.bias = bias; P.residual = residual; P.ldr = ldr; P.y = y; P.ldy = ldy;
  P.rows = rows; P.m = m; P.n = n; P.mp = L.mp; P.kblocks = (int)(L.np / LIN_BLOCK);
  P.chunks = L.G == 1 ? (int)(L.np / 32) : L.group / 32;
  P.G = (int)L.G; P.activation = activation; P.yf32 = ydtype == BAKRON_F32;
  const int64_t step = rows > 1 ? ldx : 0;      // one row may have any stride
  P.xvec = x8 ? ((uintptr_t)x | (uintptr_t)step) % 8 == 0 : aligned16(x, step * 2);
  const int ys = P.yf32 ? 4 : 2;
  P.yvec = aligned16(y, ldy * ys) && (!residual || aligned16(residual, ldr * ys));
  if (workspace && workspace_bytes >= sizeof(int) && (uintptr_t)workspace % 16 == 0) P.status = (int*)workspace;
  cudaStream_t s = (cudaStream_t)stream;
  if (rows > FEW_TOKENS) {
    const int rc = linear_tc(P, x8, L.bytes8, workspace, s);
    return rc != BAKRON_OK || !sync ? rc : bakron_read_status(workspace, stream);
  }
  if (rows <= 8)
    launch_few<1>(P, L.bytes8, x8, s);
  else
    launch_few<2>(P, L.bytes8, x8, s);
  BK_CUDA_OK(cudaGetLastError());
  if (sync) BK_CUDA_OK(cudaStreamSynchronize(s));
  return BAKRON_OK;
}
