// bakron_linear_backward: dx = dy What, the gradient of y = x What^T at the tokens x,
// What_ij = s (c_ij - z) with the grid (s, z) of row i and j's group.
//
// The sum runs over What's rows, whose scales differ, so the scale cannot wait for the end of a
// sum as it does in the forward product: an operand is s (c - z), formed in fp32 and rounded
// once to bf16.
#include <algorithm>

#include "linear.cuh"
#include "pair_gemm.cuh"

namespace bakron {
namespace {

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
    bytes = w + align256((size_t)m * ldw * 2);
  }
};

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
  BK_CUDA_OK(cudaMemsetAsync(ws, 0, sizeof(int), s));
  if (B.copy) {
    k_back_copy<<<(unsigned)std::min(rows, 8 * ROW_SMS), 256, 0, s>>>((const __nv_bfloat16*)dy, lddy, rows, m,
                                                                      (__nv_bfloat16*)(ws + B.dy), round_up(m, 8));
    BK_CUDA_OK(cudaGetLastError());
    dy = ws + B.dy;
    lddy = round_up(m, 8);
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
  CUtensorMap a, b, o;
  if (!pair_map(&a, false, dy, rows, m, rows > 1 ? lddy : round_up(m, 8), PG_K, S.a_rows) ||
      !pair_map(&b, false, E.w, m, n, B.ldw, 64, PG_K) ||
      (tma && !pair_map(&o, false, dx, rows, n, rows > 1 ? lddx : round_up(n, 8), 64, 32)))
    return BAKRON_ERR_CUDA;
  EpiBf16::Params T{tma ? nullptr : (__nv_bfloat16*)dx, lddx, rows, n, nullptr, nullptr, 0};
  BK_CUDA_OK((pair_launch<EpiBf16, false, true>(a, b, tma ? o : a, S, T, s)));
  return sync ? bakron_read_status(workspace, stream) : BAKRON_OK;
}
