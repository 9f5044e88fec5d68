// bakron_head_logprobs and bakron_head_logprobs_backward: log probabilities of given tokens
// from hidden states h (t x d) and the head's weight W (v x d), and the gradients at both,
// without the t x v logits.
//
//   l = h W^T,  lse = log sum_j exp l_j,  logp = l[target] - lse,  entropy = lse - sum_j p_j l_j
//   G_tj = dlogp ([j = target] - p_tj) - dentropy p_tj (log p_tj + entropy)
//   dh = G W,  dW = G^T h
//
// Forward: the tiles of h W^T end in the tensor cores' accumulators, and only each row's
// maximum, its sum of exponentials and that sum weighted with the logits leave them, one
// triple per row and half tile; a second kernel joins the triples in a fixed order.
//
// 1 token x 32000 x 4096 51 us (262 MB of weight at 5.1 TB/s: its rows come 128 bytes at a time), 4095 x 128256 x 4096 2.48 ms
// (1.73 PFLOP/s).
//
// Backward: the vocabulary goes in pieces.  A piece's logits are formed again, G of the
// piece is written in bf16 and multiplied by W's rows of the piece (a sum over pieces, in
// fp32) and by h (the piece's rows of dW); of up to 128 tokens in two bf16 parts.  A token's own target is no part of that bf16 G: its
// entry, often as large as all the others together and much the same from token to token, would bring its
// rounding to dh and dW.  It is kept in fp32 and joins the fp32 sums as a multiple of W's
// (h's) row.  It is formed as -g expm1(log p), as p may be nearly 1.
// 2048 x 128256 x 4096 with both gradients 3.88 ms (1.66 PFLOP/s); without dW few tokens read the
// weight twice, 64 x 50021 x 2048 96 us (G in one part 87; smaller pieces, read again from L2, 20 more).
#include <algorithm>

#include "linear.cuh"
#include "pair_gemm.cuh"

namespace bakron {
namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// What logits are taken relative to: their maximum, or 0 where that is -inf.
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
constexpr int NO_TOKEN = 0x7fffffff;

__device__ __forceinline__ float exp2_fast(float v) {      // 2 ulp, results below 2^-126 are 0
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// Column `at` of a thread's sums (written in C++ it becomes an index, and the sums local memory).
__device__ __forceinline__ float column(const float (&acc)[128], int at) {
  float l = 0.f;
#pragma unroll
  for (int u = 0; u < 128; ++u)
    asm("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, %2;\n\t@p mov.b32 %0, %3;\n\t}" : "+f"(l) : "r"(at), "r"(u), "f"(acc[u]));
  return l;
}

// ------------------------------------------------------------------ forward
// Of 2^((l - m) log2 e) over a row's half tile: the maximum m, the sum s, and x, the sum weighted
// with (l - m) log2 e.
struct EpiLse {
  struct Params {
    const int64_t* targets;
    float *m, *s, *x;      // [half tile][row]
    float* picked;         // the targets' logits
    int rows, v;
  };
  __device__ static __forceinline__ void tile(const Params& E, const PairOut& O, float (&acc)[128], const CUtensorMap*) {
    const int cols = min(O.cols, E.v - O.col);      // may be none
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < 128; ++u) {
      if (u >= cols) acc[u] = -INFINITY;
      m = max_nan(m, acc[u]);
    }
    const float base = base_of(m);
    if (O.row < E.rows && E.targets) {
      const int64_t at = E.targets[O.row] - O.col;
      if (at >= 0 && at < cols) E.picked[O.row] = column(acc, (int)at);
    }
    float s[4] = {}, x[4] = {};
#pragma unroll
    for (int u = 0; u < 128; ++u) {
      const float t = max_nan((acc[u] - base) * LOG2E, -126.f), e = exp2_fast(t);
      if (u < cols) {
        s[u & 3] += e;
        x[u & 3] = fmaf(e, t, x[u & 3]);
      }
    }
    if (O.row < E.rows) {
      const int64_t at = (int64_t)(2 * O.nt + O.half) * E.rows + O.row;
      E.m[at] = m;
      E.s[at] = (s[0] + s[1]) + (s[2] + s[3]);
      E.x[at] = (x[0] + x[1]) + (x[2] + x[3]);
    }
  }
};

static_assert(2 * PG_PAIRS <= 256, "a thread a flag");
struct JoinParams {
  const int64_t* targets;
  const float *m, *s, *x, *picked;
  int parts, rows, v;
  float *logp, *entropy, *lse;
  const int* flags;      // of the product's CTAs
  int ctas, more;        // more: not the call's first
  int* status;
};

// What the parts' triples give together: (m, s, x) of two is that of the larger maximum.
struct Triple {
  float m = -INFINITY, s = 0.f, x = 0.f;
  __device__ __forceinline__ void add(float m2, float s2, float x2) {
    const float top = max_nan(m, m2), base = base_of(top);
    const float a = max_nan((m - base) * LOG2E, -126.f), b = max_nan((m2 - base) * LOG2E, -126.f);
    const float wa = exp2_fast(a), wb = exp2_fast(b);
    x = fmaf(wa, fmaf(s, a, x), wb * fmaf(s2, b, x2));
    s = fmaf(wa, s, wb * s2);
    m = top;
  }
  __device__ __forceinline__ void warp() {      // always in the same order
#pragma unroll
    for (int o = 16; o; o >>= 1)
      add(__shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o), __shfl_xor_sync(0xffffffffu, x, o));
  }
};

__device__ __forceinline__ void head_status(const JoinParams& P) {
  if (blockIdx.x != 0) return;
  const int bad = __syncthreads_or((int)threadIdx.x < P.ctas && P.flags[threadIdx.x] != 0);
  if (threadIdx.x == 0 && (bad || !P.more)) *P.status = bad ? BAKRON_ERR_TIMEOUT : 0;
}
__device__ __forceinline__ void head_result(const JoinParams& P, const Triple& t, int row) {
  const bool none = t.m == -INFINITY;      // no logit but -inf
  const float ls = logf(t.s), lse = none ? -INFINITY : t.m + ls;
  P.lse[row] = lse;
  P.entropy[row] = none ? 0.f : ls - LN2 * (t.x / t.s);
  if (P.logp) {
    const int64_t at = P.targets[row];
    P.logp[row] = at < 0 || at >= P.v ? 0.f : none ? -INFINITY : P.picked[row] - lse;
  }
}

// Few rows: a CTA each, a thread every 512th part.
__global__ void __launch_bounds__(512) k_head_join_row(const JoinParams P) {
  __shared__ float red[3][16];
  const int row = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  head_status(P);
  Triple t;
  for (int p = threadIdx.x; p < P.parts; p += 512) {
    const int64_t at = (int64_t)p * P.rows + row;
    t.add(P.m[at], P.s[at], P.x[at]);
  }
  t.warp();
  if (lane == 0) red[0][warp] = t.m, red[1][warp] = t.s, red[2][warp] = t.x;
  __syncthreads();
  if (warp > 0) return;
  t = Triple();
  if (lane < 16) t.m = red[0][lane], t.s = red[1][lane], t.x = red[2][lane];
  t.warp();
  if (lane == 0) head_result(P, t, row);
}

// 32 rows a CTA, their triples read together: a warp takes every 32nd part, then the parts' order of a row.
__global__ void __launch_bounds__(1024) k_head_join(const JoinParams P) {
  __shared__ float red[3][32][33];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x * 32 + lane;
  pdl_wait();
  head_status(P);
  Triple t;
  if (row < P.rows) {
#pragma unroll 2
    for (int p = warp; p < P.parts; p += 32) {
      const int64_t at = (int64_t)p * P.rows + row;
      t.add(P.m[at], P.s[at], P.x[at]);
    }
  }
  red[0][warp][lane] = t.m;
  red[1][warp][lane] = t.s;
  red[2][warp][lane] = t.x;
  __syncthreads();
  t.m = red[0][lane][warp];
  t.s = red[1][lane][warp];
  t.x = red[2][lane][warp];
  t.warp();
  const int mine = blockIdx.x * 32 + warp;
  if (lane == 0 && mine < P.rows) head_result(P, t, mine);
}

// ------------------------------------------------------------------ backward
// G of a tile from its logits, summed in the forward pass's groups: a logit is then the same number there
// and here, and in l - lse, where lse is nearly the target's own logit when the model is sure of it, what
// both have lost cancels.
// TWO: G in two parts, hi in the first plane and lo in the second.
template <bool TWO>
struct EpiGrad {
  struct Params {
    const int64_t* targets;
    const float *lse, *dlogp, *entropy, *dentropy;
    float* own;      // the target's entry, where the target lies in the piece
    int rows, v, v0, count;
  };
  __device__ static __forceinline__ void tile(const Params& E, const PairOut& O, float (&acc)[128], const CUtensorMap* map) {
    float lse = 0.f, g = 0.f, u = 0.f, ent = 0.f;
    int at = -1;      // the target's column in the warp's half of the tile
    if (O.row < E.rows) {
      lse = E.lse[O.row];
      if (E.targets) {
        const int64_t target = E.targets[O.row];
        if (target >= 0 && target < E.v) {
          if (E.dlogp) g = E.dlogp[O.row];
          if (target >= E.v0 && target < (int64_t)E.v0 + E.count) at = (int)(target - E.v0) - O.col;
        }
      }
      if (E.dentropy) {
        u = E.dentropy[O.row];
        ent = E.entropy[O.row];
      }
      if (lse == -INFINITY) lse = g = u = ent = 0.f;      // no logit but -inf: zeros
    }
    if (at >= 0 && at < O.cols) {      // g (1 - p), without the difference
      const float lp = max_nan(column(acc, at) - lse, -87.f);
      E.own[O.row] = -fmaf(g, expm1f(lp), u * exp2_fast(lp * LOG2E) * (lp + ent));
    }
#pragma unroll
    for (int c = 0; c < 128; c += 64) {
      if (c >= O.cols) break;
#pragma unroll
      for (int plane = 0; plane <= (int)TWO; ++plane) {
        stage_free(O.lane);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float* z = acc + c + 8 * k + 2 * j;
            if (plane == 0) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float lp = max_nan(z[e] - lse, -87.f), p = exp2_fast(lp * LOG2E);
                z[e] = c + 8 * k + 2 * j + e == at ? 0.f : -p * fmaf(u, lp + ent, g);
              }
            }
            w[j] = bf16_pack(z[0], z[1]);
            if (TWO && plane == 0) {
              z[0] -= bf16_lo(w[j]);
              z[1] -= bf16_hi(w[j]);
            }
          }
          *staged(O.stage, O.lane, k) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        stage_ready();
        if (O.lane == 0) {
          tma_store_3d(map, O.stage, O.col + c, O.row0, plane);
          bulk_commit();
        }
      }
    }
  }
};

__global__ void __launch_bounds__(256) k_head_no_token(int* first, int* tokens, int v) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= v) return;
  first[i] = NO_TOKEN;
  tokens[i] = 0;
}
// first[j]: the first token whose target is j; tokens[j]: how many there are.
__global__ void __launch_bounds__(256) k_head_first(const int64_t* targets, int rows, int v, int* first, int* tokens) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= rows) return;
  const int64_t at = targets[i];
  if (at < 0 || at >= v) return;
  atomicMin(first + at, i);
  atomicAdd(tokens + at, 1);
}
// Row t of `more`, where t is the first token with its target and the target lies in the
// piece: the sum of own h over the tokens of that target, in their order.
constexpr int MORE_COLS = 512;
__global__ void __launch_bounds__(128) k_head_more(const int64_t* targets, const int* first, const int* tokens,
                                                   const float* own, const __nv_bfloat16* h, int64_t ldh, int rows, int d,
                                                   int v, int v0, int count, float* more, int64_t ldmore) {
  const int t = blockIdx.x, c0 = blockIdx.y * MORE_COLS + threadIdx.x;
  const int64_t target = targets[t];
  if (target < v0 || target >= (int64_t)v0 + count || target >= v || first[target] != t) return;
  __shared__ uint32_t found[2][4];
  float acc[4] = {};
  int left = tokens[target];      // (a target that is not repeated is found at once)
  for (int i0 = t, turn = 0; i0 < rows && left > 0; i0 += 128, turn ^= 1) {
    const int i = i0 + threadIdx.x;
    const uint32_t same = __ballot_sync(0xffffffffu, i < rows && targets[i] == target);
    if ((threadIdx.x & 31) == 0) found[turn][threadIdx.x >> 5] = same;
    __syncthreads();
    for (int w = 0; w < 4; ++w)
      for (uint32_t bits = found[turn][w]; bits; bits &= bits - 1, --left) {
        const int at = i0 + 32 * w + __ffs((int)bits) - 1;
        const float a = own[at];
        const __nv_bfloat16* row = h + at * ldh;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c0 + 128 * k < d) acc[k] = fmaf(a, __bfloat162float(row[c0 + 128 * k]), acc[k]);
      }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (c0 + 128 * k < d) more[(int64_t)t * ldmore + c0 + 128 * k] = acc[k];
}

// dh = the parts' sum (with two parts of G: of both) + own W[target], rounded once.  A thread has 4 columns.
__global__ void __launch_bounds__(256) k_head_dh(const float* part, int splits, int planes, int64_t ldp, const int64_t* targets,
                                                 const float* own, const __nv_bfloat16* w, int64_t ldw, int rows,
                                                 int d, int v, __nv_bfloat16* dh, int64_t lddh, int vec) {
  pdl_wait();
  const int row = blockIdx.x;
  const int64_t target = targets ? targets[row] : -1;
  const bool scored = target >= 0 && target < v;
  const float a = scored ? own[row] : 0.f;
  for (int c = (blockIdx.y * 256 + threadIdx.x) * 4; c < d; c += 1024 * gridDim.y) {
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* from = part + row * ldp + c;      // (its rows are whole float4s)
#pragma unroll 4
    for (int s = 0; s < splits * planes; ++s) {
      const float4 u = *reinterpret_cast<const float4*>(from + (int64_t)s * rows * ldp);
      sum.x += u.x;
      sum.y += u.y;
      sum.z += u.z;
      sum.w += u.w;
    }
    float o[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (scored && c + k < d) o[k] = fmaf(a, __bfloat162float(w[target * ldw + c + k]), o[k]);
    __nv_bfloat16* out = dh + row * lddh + c;
    if (vec && c + 4 <= d) {
      *reinterpret_cast<uint2*>(out) = make_uint2(bf16_pack(o[0], o[1]), bf16_pack(o[2], o[3]));
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + k < d) out[k] = __float2bfloat16_rn(o[k]);
    }
  }
}

// h one below the other, for the two parts of G.
__global__ void __launch_bounds__(256) k_head_twice(const __nv_bfloat16* h, int64_t ldh, int rows, int d, __nv_bfloat16* to, int64_t ldt) {
  const __nv_bfloat16* from = h + (int64_t)(blockIdx.x % rows) * ldh;
  for (int c = blockIdx.y * 256 + threadIdx.x; c < d; c += 256 * gridDim.y) to[blockIdx.x * ldt + c] = from[c];
}

// ------------------------------------------------------------------ host side
constexpr int HEAD_MAX_ROWS = 1 << 24, HEAD_MAX_V = 1 << 24, HEAD_MAX_D = 1 << 16;
constexpr int LSE_ROWS = 16384;        // tokens of one forward pass over the weight: bounds the triples
// K blocks (512 values) summed in place: in the tensor cores a sum is cut, not rounded, at each of its
// additions.  2048 x 32768 x 4096 in place all the way 294 us and lse up to 3.8e-5 off, so 300 and 3.5e-6.
constexpr int LSE_GROUP = 8;
constexpr int64_t G_BYTES = 256 << 20; // of G kept at a time
// Tokens up to which G is kept in two bf16 parts, rows one below the other: they fill a tile's rows, which cost nothing.  In one
// part its rounding is as large as a result's own; over many tokens and a large vocabulary it averages out beside
// the targets' entries, and two parts would take 3/5 more time.
constexpr int TWO_PARTS = PG_M / 2;

bool head_ok(int rows, int v, int d) {
  return rows >= 0 && rows <= HEAD_MAX_ROWS && v >= 1 && v <= HEAD_MAX_V && d >= 1 && d <= HEAD_MAX_D;
}
bool in_place(const void* p, int64_t rows, int64_t ld) { return aligned16(p, rows > 1 ? ld * 2 : 0); }
// The row stride a tensor map gets (any, for a single row).
int64_t map_ld(int64_t rows, int64_t ld, int d) { return rows > 1 ? ld : round_up(d, 8); }

// Columns of a tile for few tokens: as few as the busiest pair can get (1 token x 32000 x 4096: 224
// columns 51 us, 256 54).
int lse_bn(int rows, int v) {
  if (rows > PG_M) return 256;
  int best = 256;
  int64_t cost = INT64_MAX;
  for (int bn = 256; bn >= 128; bn -= 32) {
    const int64_t c = (int64_t)ceil_div(ceil_div(v, bn), PG_PAIRS) * bn;
    if (c < cost) {
      cost = c;
      best = bn;
    }
  }
  return best;
}

int box_rows(int rows) { return rows >= 128 ? 128 : (int)round_up(rows, 8); }

// Offsets into the workspaces.
struct Carve {
  size_t at = 256;
  size_t take(size_t bytes) {
    const size_t r = at;
    at += align256(bytes);
    return r;
  }
};
struct HeadLayout {
  size_t flags, h = 0, w = 0, m, s, x, picked, bytes;
  bool copy_h, copy_w;
  HeadLayout(const void* ph, int64_t ldh, const void* pw, int64_t ldw, int rows, int v, int d) {
    Carve c;
    flags = c.take(2 * PG_PAIRS * sizeof(int));
    copy_h = !in_place(ph, rows, ldh);
    copy_w = !in_place(pw, v, ldw);
    if (copy_h) h = c.take((size_t)rows * round_up(d, 8) * 2);
    if (copy_w) w = c.take((size_t)v * round_up(d, 8) * 2);
    const int slice = std::min(rows, LSE_ROWS);
    const size_t triples = (size_t)2 * ceil_div(v, lse_bn(slice, v)) * slice * 4;
    m = c.take(triples);
    s = c.take(triples);
    x = c.take(triples);
    picked = c.take((size_t)slice * 4);
    bytes = c.at;
  }
};
struct HeadBackLayout {
  size_t h = 0, w = 0, twice = 0, own, first = 0, tokens = 0, more = 0, g, part, bytes;
  bool copy_h, copy_w;
  int planes, piece, splits;      // parts of G
  int64_t ldg, ldp;      // of G, and of the fp32 sums
  HeadBackLayout(const void* ph, int64_t ldh, const void* pw, int64_t ldw, int rows, int v, int d, bool dw) {
    Carve c;
    copy_h = !in_place(ph, rows, ldh);
    copy_w = !in_place(pw, v, ldw);
    if (copy_h) h = c.take((size_t)rows * round_up(d, 8) * 2);
    if (copy_w) w = c.take((size_t)v * round_up(d, 8) * 2);
    planes = rows <= TWO_PARTS ? 2 : 1;
    if (dw && planes == 2) twice = c.take((size_t)2 * rows * round_up(d, 8) * 2);
    const int64_t most = std::max<int64_t>(256, G_BYTES / 2 / std::max(planes * rows, 1) / 256 * 256);
    const int pieces = (int)((v + most - 1) / most);
    piece = (int)std::min<int64_t>(v, round_up(ceil_div(v, pieces), 256));
    ldg = round_up(piece, 8);
    ldp = round_up(d, 4);
    // dh's sum runs over the piece in `splits` ranges: what the busiest pair takes, a range costing
    // some 4 blocks beside its own (2048 tokens x 128256 x 4096 by 2 ranges 4.00 ms forward and back, by 4 3.86)
    const int64_t tiles = (int64_t)ceil_div(planes * rows, PG_M) * ceil_div(d, 256);
    const int nk = ceil_div(piece, PG_K);
    auto cost = [&](int s) { return (tiles * s + PG_PAIRS - 1) / PG_PAIRS * (ceil_div(nk, s) + 4); };
    splits = 1;
    for (int s = 2; s <= std::min(32, nk); ++s)
      if (cost(s) * 50 < cost(splits) * 49) splits = s;
    own = c.take((size_t)rows * 4);
    if (dw) {
      first = c.take((size_t)v * 4);
      tokens = c.take((size_t)v * 4);
      more = c.take((size_t)rows * ldp * 4);
    }
    g = c.take((size_t)planes * rows * ldg * 2);
    part = c.take((size_t)splits * planes * rows * ldp * 4);
    bytes = c.at;
  }
};

PairShape head_shape(int rows, int bn, int tn, int nk, int* status) {
  PairShape S{};
  S.tm = ceil_div(rows, PG_M);
  S.tn = tn;
  S.bn = bn;
  S.nk = S.per = nk;
  S.splits = 1;
  S.group = PG_GROUP;
  S.band = 16;
  S.rows = rows;
  S.a_rows = box_rows(rows);
  S.status = status;
  S.spin_cycles = spin_cycles_from_env();
  return S;
}

}  // namespace
}  // namespace bakron

using namespace bakron;

extern "C" size_t bakron_head_logprobs_workspace_bytes(const void* h, int64_t ldh, const void* weight, int64_t ldw,
                                                       int rows, int v, int d) {
  return head_ok(rows, v, d) && rows > 0 ? HeadLayout(h, ldh, weight, ldw, rows, v, d).bytes : 0;
}

extern "C" int bakron_head_logprobs(const void* h, int64_t ldh, const void* weight, int64_t ldw, int rows, int v, int d,
                                    const int64_t* targets, float* logp, float* entropy, float* lse, void* workspace,
                                    size_t workspace_bytes, int sync, void* stream) {
  if (!head_ok(rows, v, d)) return BAKRON_ERR_INVALID_ARG;
  if (rows == 0) return BAKRON_OK;
  if (!h || !weight || ldh < d || ldw < d || !entropy || !lse || (targets && !logp) || (!targets && logp) || !workspace ||
      (uintptr_t)workspace % 16 != 0 || (uintptr_t)h % 2 != 0 || (uintptr_t)weight % 2 != 0)
    return BAKRON_ERR_INVALID_ARG;
  const HeadLayout L(h, ldh, weight, ldw, rows, v, d);
  if (workspace_bytes < L.bytes) return BAKRON_ERR_WORKSPACE;
  cudaStream_t s = (cudaStream_t)stream;
  char* ws = (char*)workspace;
  if (L.copy_h) {
    BK_CUDA_OK(pair_copy(h, ldh, rows, d, ws + L.h, s));
    h = ws + L.h;
    ldh = round_up(d, 8);
  }
  if (L.copy_w) {
    BK_CUDA_OK(pair_copy(weight, ldw, v, d, ws + L.w, s));
    weight = ws + L.w;
    ldw = round_up(d, 8);
  }
  for (int r0 = 0; r0 < rows; r0 += LSE_ROWS) {
    const int n = std::min(rows - r0, LSE_ROWS), bn = lse_bn(std::min(rows, LSE_ROWS), v);
    PairShape S = head_shape(n, bn, ceil_div(v, bn), ceil_div(d, PG_K), (int*)ws);
    S.group = LSE_GROUP;
    S.flags = (int*)(ws + L.flags);
    CUtensorMap a, b;
    if (!pair_map(&a, false, (const __nv_bfloat16*)h + r0 * ldh, n, d, map_ld(n, ldh, d), PG_K, S.a_rows) ||
        !pair_map(&b, false, weight, v, d, map_ld(v, ldw, d), PG_K, bn / 2))
      return BAKRON_ERR_CUDA;
    EpiLse::Params E{targets ? targets + r0 : nullptr, (float*)(ws + L.m), (float*)(ws + L.s), (float*)(ws + L.x),
                     (float*)(ws + L.picked), n, v};
    BK_CUDA_OK((pair_launch<EpiLse, false, false>(a, b, b, S, E, s)));
    JoinParams J{E.targets, E.m, E.s, E.x, E.picked, 2 * S.tn, n, v, logp ? logp + r0 : nullptr, entropy + r0, lse + r0,
                 S.flags, (int)pair_ctas(S), r0 > 0, (int*)ws};
    BK_CUDA_OK(n < 64 ? launch_pdl(k_head_join_row, dim3(n), dim3(512), 0, s, J)
                      : launch_pdl(k_head_join, dim3(ceil_div(n, 32)), dim3(1024), 0, s, J));
  }
  return sync ? bakron_read_status(workspace, stream) : BAKRON_OK;
}

extern "C" size_t bakron_head_logprobs_backward_workspace_bytes(const void* h, int64_t ldh, const void* weight,
                                                                int64_t ldw, int rows, int v, int d, int weight_grad) {
  return head_ok(rows, v, d) && rows > 0 ? HeadBackLayout(h, ldh, weight, ldw, rows, v, d, weight_grad != 0).bytes : 0;
}

extern "C" int bakron_head_logprobs_backward(const void* h, int64_t ldh, const void* weight, int64_t ldw, int rows,
                                             int v, int d, const int64_t* targets, const float* lse,
                                             const float* dlogp, const float* entropy, const float* dentropy, void* dh,
                                             int64_t lddh, void* dweight, int64_t lddw, void* workspace,
                                             size_t workspace_bytes, int sync, void* stream) {
  if (!head_ok(rows, v, d)) return BAKRON_ERR_INVALID_ARG;
  if ((dweight && lddw < d) || (rows > 0 && (!h || !weight || ldh < d || ldw < d || !lse || (dlogp && !targets) ||
                                             (dentropy && !entropy) || !dh || lddh < d || !workspace ||
                                             (uintptr_t)workspace % 16 != 0 || (uintptr_t)h % 2 != 0 ||
                                             (uintptr_t)weight % 2 != 0)))
    return BAKRON_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  if (rows == 0) {      // no token: no gradient at the weight
    if (dweight) BK_CUDA_OK(cudaMemset2DAsync(dweight, (size_t)lddw * 2, 0, (size_t)d * 2, (size_t)v, s));
    if (sync) BK_CUDA_OK(cudaStreamSynchronize(s));
    return BAKRON_OK;
  }
  const HeadBackLayout L(h, ldh, weight, ldw, rows, v, d, dweight != nullptr);
  if (workspace_bytes < L.bytes) return BAKRON_ERR_WORKSPACE;
  char* ws = (char*)workspace;
  k_clear_status<<<1, 1, 0, s>>>((int*)ws);
  BK_CUDA_OK(cudaGetLastError());
  if (L.copy_h) {
    BK_CUDA_OK(pair_copy(h, ldh, rows, d, ws + L.h, s));
    h = ws + L.h;
    ldh = round_up(d, 8);
  }
  if (L.copy_w) {
    BK_CUDA_OK(pair_copy(weight, ldw, v, d, ws + L.w, s));
    weight = ws + L.w;
    ldw = round_up(d, 8);
  }
  float *own = (float*)(ws + L.own), *more = (float*)(ws + L.more), *part = (float*)(ws + L.part);
  int *first = (int*)(ws + L.first), *tokens = (int*)(ws + L.tokens);
  const bool near = dweight && targets && dlogp;      // dW gets the targets' rows
  if (near) {
    k_head_no_token<<<ceil_div(v, 256), 256, 0, s>>>(first, tokens, v);
    k_head_first<<<ceil_div(rows, 256), 256, 0, s>>>(targets, rows, v, first, tokens);
    BK_CUDA_OK(cudaGetLastError());
  }
  const int grows = L.planes * rows;      // rows of G
  const void* hg = h;                     // h for them
  int64_t ldhg = ldh;
  if (dweight && L.planes == 2) {
    hg = ws + L.twice;
    ldhg = round_up(d, 8);
    k_head_twice<<<dim3((unsigned)grows, (unsigned)std::min(ceil_div(d, 512), 16)), 256, 0, s>>>((const __nv_bfloat16*)h, ldh, rows, d,
                                                                                             (__nv_bfloat16*)hg, ldhg);
    BK_CUDA_OK(cudaGetLastError());
  }
  const bool dw_tma = dweight && in_place(dweight, v, lddw);
  for (int v0 = 0; v0 < v; v0 += L.piece) {
    const int count = std::min(v - v0, L.piece);
    const __nv_bfloat16* w = (const __nv_bfloat16*)weight + v0 * ldw;
    void* G = ws + L.g;
    CUtensorMap a, b, o;
    // G of the piece
    PairShape S = head_shape(rows, 256, ceil_div(count, 256), ceil_div(d, PG_K), (int*)ws);
    S.group = LSE_GROUP;
    if (!pair_map(&a, false, h, rows, d, map_ld(rows, ldh, d), PG_K, S.a_rows) ||
        !pair_map(&b, false, w, count, d, map_ld(count, ldw, d), PG_K, 128) ||
        !pair_map(&o, false, G, rows, count, L.ldg, 64, 32, L.planes))
      return BAKRON_ERR_CUDA;
    auto g_of_piece = [&](auto epi) -> cudaError_t {
      using Epi = decltype(epi);
      const typename Epi::Params E{dlogp ? targets : nullptr, lse, dlogp, entropy, dentropy, own, rows, v, v0, count};
      return pair_launch<Epi, false, false>(a, b, o, S, E, s);
    };
    BK_CUDA_OK(L.planes == 2 ? g_of_piece(EpiGrad<true>()) : g_of_piece(EpiGrad<false>()));
    // dh's part
    S = head_shape(grows, 256, ceil_div(d, 256), ceil_div(count, PG_K), (int*)ws);
    S.splits = L.splits;
    S.per = ceil_div(S.nk, S.splits);
    S.splits = ceil_div(S.nk, S.per);
    if (!pair_map(&a, false, G, grows, count, L.ldg, PG_K, S.a_rows) ||
        !pair_map(&b, false, w, count, d, map_ld(count, ldw, d), 64, PG_K) ||
        !pair_map(&o, true, part, grows, d, L.ldp, 32, 32, L.splits))
      return BAKRON_ERR_CUDA;
    if (S.splits < L.splits && v0 == 0)      // no part of the rest: zeros
      BK_CUDA_OK(cudaMemsetAsync(part + (int64_t)S.splits * grows * L.ldp, 0,
                                 (size_t)(L.splits - S.splits) * grows * L.ldp * 4, s));
    BK_CUDA_OK((pair_launch<EpiF32, false, true>(a, b, o, S, EpiF32::Params{v0 > 0}, s)));
    if (!dweight) continue;
    // the piece's rows of dW
    if (near) {
      k_head_more<<<dim3((unsigned)rows, (unsigned)ceil_div(d, MORE_COLS)), 128, 0, s>>>(
          targets, first, tokens, own, (const __nv_bfloat16*)h, ldh, rows, d, v, v0, count, more, L.ldp);
      BK_CUDA_OK(cudaGetLastError());
    }
    __nv_bfloat16* c = (__nv_bfloat16*)dweight + v0 * lddw;
    S = head_shape(count, 256, ceil_div(d, 256), ceil_div(grows, PG_K), (int*)ws);
    S.band = 8;
    if (!pair_map(&a, false, G, grows, count, L.ldg, 64, PG_K) ||
        !pair_map(&b, false, hg, grows, d, map_ld(grows, ldhg, d), 64, PG_K) ||
        (dw_tma && !pair_map(&o, false, c, count, d, map_ld(count, lddw, d), 64, 32)))
      return BAKRON_ERR_CUDA;
    EpiBf16::Params B{dw_tma ? nullptr : c, lddw, count, d, near ? first + v0 : nullptr, more, L.ldp};
    BK_CUDA_OK((pair_launch<EpiBf16, true, true>(a, b, dw_tma ? o : a, S, B, s)));
  }
  BK_CUDA_OK(launch_pdl(k_head_dh, dim3((unsigned)rows, (unsigned)std::min(ceil_div(d, 1024), 8)), dim3(256), 0, s, part,
                        L.splits, L.planes, L.ldp, dlogp ? targets : nullptr, own, (const __nv_bfloat16*)weight, ldw, rows, d, v,
                        (__nv_bfloat16*)dh, lddh, (int)(((uintptr_t)dh | (uintptr_t)(rows > 1 ? lddh * 2 : 0)) % 8 == 0)));
  return sync ? bakron_read_status(workspace, stream) : BAKRON_OK;
}
