// A linear layer with its epilogue, and what its backward needs besides two plain products:
//
//   z = x W^T + bias,  y = act(z) + residual
//   dz = dy act'(z),   dbias = sum_m dz,   dx = dz W,   dW = dz^T x
//
// The accumulator stays in fp32 through bias, activation and residual; y (and z, where it is kept for the
// backward) are rounded once, when they are stored.  dz is rounded to bf16 because it is an operand of the two
// products; dbias sums the unrounded values.
//
// Large M: pair tiles on the tensor cores (pair_tile_sm100.cuh), bound by the MMAs; bias, activation,
// residual and the stores of a tile run under the next tile's MMAs.  Few rows: linear_rows_kernel, bound by
// reading W once.
#pragma once

#include "norm_kernels.cuh"
#include "pair_tile_sm100.cuh"

namespace npd {

enum : int { kActNone = 0, kActRelu, kActGelu, kActGeluTanh, kActSilu, kActCount };

constexpr float kGeluK = 0.797884560802865355880f;  // sqrt(2 / pi)
constexpr float kGeluC = 0.044715f;
constexpr float kLog2e = 1.442695040888963407360f;

// 1 / (1 + e^-v); exact limits at both ends (e^-v overflows to infinity, whose reciprocal is 0).
__device__ __forceinline__ float sigmoidf(float v) { return __fdividef(1.f, 1.f + ex2f(-kLog2e * v)); }

// e^(-z^2 / 2), off by 2 z^2 + 4 units of 2^-24 relative to the value.
__device__ __forceinline__ float gauss(float z) { return ex2f((-0.5f * kLog2e * z) * z); }

// Normal distribution function from e = gauss(z): Phi(-a) = e t (c0 + c1 t + ... + c7 t^7), t = 1 / (1 + 0.305 a), a >= 0.
// The coefficients are a fit of our own, the least largest relative error over 0 <= a <= 14.5 (1.0e-7, by Lawson's weighted
// least squares), so the tail is right relative to its own size, not to 1: GELU at z = -6 is about 6e-9, and a fit that
// is good to 1.5e-7 absolutely leaves it off by 0.4 %, at z = -8 by 1 %.  With the roundings: (2 z^2 + 32) 2^-24
// relative, down to where e leaves the normal range (z = -13).  Two special-function instructions and twelve others; the
// library's erfcf made the epilogue of a K = 1536 tile take three times as long as its MMAs.
__device__ __forceinline__ float normal_cdf(float z, float e) {
  const float t = __fdividef(1.f, fmaf(0.305000007f, fabsf(z), 1.f));
  float s = fmaf(0.0366388485f, t, -0.152746022f);
  s = fmaf(s, t, 0.185314819f);
  s = fmaf(s, t, -0.0376205817f);
  s = fmaf(s, t, 0.120840348f);
  s = fmaf(s, t, 0.103473708f);
  s = fmaf(s, t, 0.122458681f);
  s = fmaf(s, t, 0.121640243f);
  const float q = s * t * e;  // Phi(-|z|)
  return z < 0.f ? q : 1.f - q;
}

__device__ __forceinline__ float act_value(int act, float z) {
  switch (act) {
    case kActRelu: return z < 0.f ? 0.f : z;  // NaN stays NaN
    case kActGelu: return z * normal_cdf(z, gauss(z));
    case kActGeluTanh: return z * sigmoidf(2.f * kGeluK * z * fmaf(kGeluC, z * z, 1.f));  // (1 + tanh u) / 2 = 1 / (1 + e^-2u)
    case kActSilu: return z * sigmoidf(z);
    default: return z;
  }
}
__device__ __forceinline__ float act_slope(int act, float z) {
  switch (act) {
    case kActRelu: return z > 0.f ? 1.f : 0.f;
    case kActGelu: {
      const float e = gauss(z);
      return fmaf(0.398942280401432677940f * z, e, normal_cdf(z, e));  // Phi(z) + z phi(z)
    }
    case kActGeluTanh: {
      // q (1 - q) is 0 long before |z| = 100; what multiplies it stays finite, since 0 * inf is not 0
      const float zc = fminf(fmaxf(z, -100.f), 100.f), z2 = zc * zc;
      const float q = sigmoidf(2.f * kGeluK * z * fmaf(kGeluC, z2, 1.f));
      return fmaf(2.f * zc * q * (1.f - q) * kGeluK, fmaf(3.f * kGeluC, z2, 1.f), q);
    }
    case kActSilu: {
      const float s = sigmoidf(z);
      return s * fmaf(z, 1.f - s, 1.f);
    }
    default: return 1.f;
  }
}

struct LinearParams {
  int M, N, K, ksteps;
  int act;
  const __nv_bfloat16* x;       // linear_rows_kernel only (the tiles read through tensor maps)
  const __nv_bfloat16* w;
  long long ldx, ldw;
  const void* bias;             // [N] or NULL
  int bias_f32;
  const void* residual;         // y's type [M, ldr] or NULL
  long long ldr;
  void* y;
  __nv_bfloat16* z;             // or NULL
  long long ldy, ldz;
  int y_f32;                    // linear_rows_kernel only: y and residual are fp32
  int wide_y, wide_z;           // every row starts on a 32-byte boundary
  int mtiles, ntiles, group;    // tiles of 256 x kBN; rows of tiles per group (see LinearWalk)
  int* status;
};

__device__ __forceinline__ float linear_bias(const LinearParams& p, int n) {
  return p.bias_f32 ? static_cast<const float*>(p.bias)[n] : __bfloat162float(static_cast<const __nv_bfloat16*>(p.bias)[n]);
}

// Tiles dealt round robin, in groups of rows of tiles whose x fits a quarter of L2; within a group the
// row of tiles varies fastest: pairs that work at the same time share W tiles, and x stays in L2.
struct LinearWalk {
  int mtiles, ntiles, group, v, step;
  __device__ __forceinline__ LinearWalk(const LinearParams& p, int pair, int pairs)
      : mtiles(p.mtiles), ntiles(p.ntiles), group(p.group), v(pair - pairs), step(pairs) {}
  __device__ __forceinline__ bool next(PairTile& t) {
    v += step;
    if (v >= mtiles * ntiles) return false;
    const int per = group * ntiles, g = v / per, local = v - g * per;
    const int rows = min(group, mtiles - g * group);
    t.tile = local / rows;
    t.row0 = 256 * (g * group + local % rows);
    t.run = 0;
    t.first = t.last = true;
    return true;
  }
};

// kY32: y and residual are fp32.  kKeepZ: z is stored too.
template <bool kY32, bool kKeepZ, int kTileN>
struct LinearEpi {
  using Params = LinearParams;
  using Walk = LinearWalk;
  static constexpr int kBN = kTileN, kGroupN = PairCfg<kBN>::BNG;
  static __device__ __forceinline__ int rows(const Params& p) { return p.M; }
  const Params& p;
  int pair_row, group, lane, row;
  uint4 next[kY32 ? 8 : 4];  // residual of the next chunk: its loads run under the chunk before
  float bias[2];             // of this lane's column in either chunk
  __device__ __forceinline__ LinearEpi(const Params& p_, int pair_row_, int group_)
      : p(p_), pair_row(pair_row_), group(group_), lane(threadIdx.x & 31), row(0), bias{0.f, 0.f} {}
  __device__ __forceinline__ void fetch(int col0) {
    constexpr int kE = kY32 ? 4 : 2, kPerVec = 16 / kE, kVecs = 32 / kPerVec;
    if (p.residual == nullptr || row >= p.M) return;
    const char* src = static_cast<const char*>(p.residual) + (static_cast<size_t>(row) * p.ldr + col0) * kE;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int c = col0 + i * kPerVec;
      next[i] = make_uint4(0u, 0u, 0u, 0u);
      if (c + kPerVec <= p.N) {
        next[i] = *reinterpret_cast<const uint4*>(src + 16 * i);
      } else if (c < p.N) {  // the row ends inside this vector
        uint32_t w[4] = {0u, 0u, 0u, 0u};
        for (int k = 0; k < kPerVec; ++k) {
          if (c + k >= p.N) break;
          if (kY32) w[k & 3] = reinterpret_cast<const uint32_t*>(src + 16 * i)[k];
          else w[(k >> 1) & 3] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(src + 16 * i)[k]) << (16 * (k & 1));
        }
        next[i] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
  __device__ __forceinline__ void begin(const PairTile& t) {
    row = t.row0 + pair_row;
    const int col0 = t.tile * kBN + group * kGroupN;
    if (col0 < p.N) fetch(col0);
    if (p.bias != nullptr) {
#pragma unroll
      for (int i = 0; i < kGroupN / 32; ++i) bias[i] = col0 + 32 * i + lane < p.N ? linear_bias(p, col0 + 32 * i + lane) : 0.f;
    }
  }
  __device__ __forceinline__ void chunk(const uint32_t (&acc)[32], int col0) {
    const int n = p.N - col0;
    if (n <= 0) return;  // the same for the whole warp
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(acc[i]);
    if (p.bias != nullptr) {
      // loaded once per warp, a column per lane, and handed round by shuffles
      const float b = col0 % kGroupN == 0 ? bias[0] : bias[1];
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] += __shfl_sync(0xffffffffu, b, i);
    }
    if (kKeepZ && row < p.M) store_row32<false>(p.z + static_cast<size_t>(row) * p.ldz + col0, v, n, p.wide_z != 0);
    switch (p.act) {  // the same for the whole grid
      case kActRelu: apply<kActRelu>(v); break;
      case kActGelu: apply<kActGelu>(v); break;
      case kActGeluTanh: apply<kActGeluTanh>(v); break;
      case kActSilu: apply<kActSilu>(v); break;
      default: break;
    }
    if (p.residual != nullptr && row < p.M) {
#pragma unroll
      for (int i = 0; i < (kY32 ? 8 : 4); ++i) {
        const uint32_t w[4] = {next[i].x, next[i].y, next[i].z, next[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (kY32) {
            v[(4 * i + k) & 31] += __uint_as_float(w[k]);
          } else {
            v[(8 * i + 2 * k) & 31] += bf16_lo(w[k]);
            v[(8 * i + 2 * k + 1) & 31] += bf16_hi(w[k]);
          }
        }
      }
      const int last = (col0 / kGroupN + 1) * kGroupN;  // end of this group's columns
      if (col0 + 32 < min(last, p.N)) fetch(col0 + 32);
    }
    if (row < p.M)
      store_row32<kY32>(static_cast<char*>(p.y) + (static_cast<size_t>(row) * p.ldy + col0) * (kY32 ? 4 : 2), v, n, p.wide_y != 0);
  }
  template <int kAct>
  static __device__ __forceinline__ void apply(float (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = act_value(kAct, v[i]);
  }
  __device__ __forceinline__ void end(const PairTile&) {}
};

// ---------------------------------------------------------------------------------------------
// Few rows (one decoded token to kRowsMax): every weight is used a handful of times, so the floor is reading W
// once.  It is reached as far as there are blocks to read it (one row, from HBM: N = 6144, K = 1536 6.8 us against 2.9 of bytes;
// N = 1536, K = 6144, 96 blocks on 148 SMs, 11.4, with W already in L2 6.2; N = 16,384, K = 4096 24 against 20.5; 32 rows
// at the last two 21 and 53 us: x is read again by every block, and nothing is loaded ahead of the batch in use).  A block takes
// 16 rows of W; its warps share out K and add their parts up in shared
// memory, in a fixed order.  mma.sync m16n8k16 with W as the 16-row operand and the tokens as its 8
// columns: the tensor throughput does not matter here, and this form takes the operands straight from
// global memory to registers, without staging (tcgen05 reads its operands from shared memory): the order
// of the contraction is free, so a thread's 16-byte vector of a row serves as the k indices that the
// instruction gives this thread in two successive MMAs, for W and x alike.
// ---------------------------------------------------------------------------------------------
namespace rows_cfg {
constexpr int kRowsMax = 32;
constexpr int kWarps = 8, kUnroll = 4;
}  // namespace rows_cfg

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// kG groups of 8 tokens.
template <int kG>
__global__ void __launch_bounds__(32 * rows_cfg::kWarps) linear_rows_kernel(const LinearParams p) {
  using namespace rows_cfg;
  __shared__ float part[kWarps][kG * 8][17];  // [warp][token][row of W], padded against bank conflicts
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, q = lane & 3;
  const int n0 = blockIdx.x * 16;
  grid_dependency_wait();
  grid_launch_dependents();
  const __nv_bfloat16* w0 = p.w + static_cast<size_t>(min(n0 + g, p.N - 1)) * p.ldw;      // rows beyond N: computed
  const __nv_bfloat16* w1 = p.w + static_cast<size_t>(min(n0 + g + 8, p.N - 1)) * p.ldw;  // from the last one, not stored
  const __nv_bfloat16* xr[kG];
#pragma unroll
  for (int i = 0; i < kG; ++i) xr[i] = p.x + static_cast<size_t>(min(8 * i + g, p.M - 1)) * p.ldx;
  float acc[kG][4];
#pragma unroll
  for (int i = 0; i < kG; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
  // steps of 32 along K, dealt to the warps in contiguous stretches
  const int steps = (p.K + 31) / 32;
  const int s0 = static_cast<int>(static_cast<long long>(steps) * warp / kWarps);
  const int s1 = static_cast<int>(static_cast<long long>(steps) * (warp + 1) / kWarps);
  const int full = min(s1, p.K / 32);  // steps before this one lie inside K
  auto multiply = [&](const uint4& a, const uint4& b, const uint4 (&x)[kG]) {
#pragma unroll
    for (int i = 0; i < kG; ++i) {
      mma_16816(acc[i], a.x, b.x, a.y, b.y, x[i].x, x[i].y);
      mma_16816(acc[i], a.z, b.z, a.w, b.w, x[i].z, x[i].w);
    }
  };
  int s = s0;
  for (; s + kUnroll <= full; s += kUnroll) {
    uint4 a[kUnroll], b[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int k = (s + u) * 32 + 8 * q;
      a[u] = __ldg(reinterpret_cast<const uint4*>(w0 + k));
      b[u] = __ldg(reinterpret_cast<const uint4*>(w1 + k));
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int k = (s + u) * 32 + 8 * q;
      uint4 x[kG];
#pragma unroll
      for (int i = 0; i < kG; ++i) x[i] = __ldg(reinterpret_cast<const uint4*>(xr[i] + k));
      multiply(a[u], b[u], x);
    }
  }
  for (; s < s1; ++s) {
    const int k = s * 32 + 8 * q;
    const uint4 a = load8<false>(w0, k, p.K).q[0], b = load8<false>(w1, k, p.K).q[0];
    uint4 x[kG];
#pragma unroll
    for (int i = 0; i < kG; ++i) x[i] = load8<false>(xr[i], k, p.K).q[0];
    multiply(a, b, x);
  }
#pragma unroll
  for (int i = 0; i < kG; ++i) {
    part[warp][8 * i + 2 * q][g] = acc[i][0];
    part[warp][8 * i + 2 * q + 1][g] = acc[i][1];
    part[warp][8 * i + 2 * q][g + 8] = acc[i][2];
    part[warp][8 * i + 2 * q + 1][g + 8] = acc[i][3];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * p.M; i += blockDim.x) {
    const int m = i >> 4, r = i & 15, n = n0 + r;
    if (n >= p.N) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += part[w][m][r];
    if (p.bias != nullptr) v += linear_bias(p, n);
    if (p.z != nullptr) p.z[static_cast<size_t>(m) * p.ldz + n] = __float2bfloat16_rn(v);
    v = act_value(p.act, v);
    const size_t at = static_cast<size_t>(m) * p.ldy + n, rt = static_cast<size_t>(m) * p.ldr + n;
    if (p.y_f32) {
      if (p.residual != nullptr) v += static_cast<const float*>(p.residual)[rt];
      static_cast<float*>(p.y)[at] = v;
    } else {
      if (p.residual != nullptr) v += __bfloat162float(static_cast<const __nv_bfloat16*>(p.residual)[rt]);
      static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(v);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// dz = dy act'(z) in bf16 (left out without an activation) and, per block of rows, the column sums of the
// unrounded dz.  A warp covers 256 columns, eight per lane; the block's 8 warps take every 8th row.
// ---------------------------------------------------------------------------------------------
struct LinearGradParams {
  int M, N, act, rows_per_block;
  const __nv_bfloat16* dy;
  const __nv_bfloat16* z;
  __nv_bfloat16* dz;     // or NULL
  long long lddy, ldz, lddz, ldpart;
  float* part;           // [gridDim.y][ldpart] or NULL
};

// kRagged: N need not be a multiple of 8.  Four blocks of 64 registers per SM: with six of 40 the loop keeps less in
// flight (M = 8192, N = 16,384 and a dx product of K = 64: GELU 268 us instead of 292, its tanh form 259 instead of 287).
template <int kAct, bool kRagged>
__global__ void __launch_bounds__(256, 4) linear_dz_kernel(const LinearGradParams p) {
  __shared__ float sums[8][256 + 8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 256 + lane * 8;
  const int m0 = blockIdx.y * p.rows_per_block, m1 = min(p.M, m0 + p.rows_per_block);
  grid_dependency_wait();
  V8 s;
#pragma unroll
  for (int i = 0; i < 8; ++i) s.v[i] = 0.f;
  if (c < p.N) {
    // the next row's loads are in flight while this row's slopes are evaluated
    const int n = p.N - c;
    const __nv_bfloat16* pd = p.dy + static_cast<size_t>(m0 + warp) * p.lddy + c;
    const __nv_bfloat16* pz = kAct != kActNone ? p.z + static_cast<size_t>(m0 + warp) * p.ldz + c : nullptr;
    __nv_bfloat16* po = kAct != kActNone ? p.dz + static_cast<size_t>(m0 + warp) * p.lddz : nullptr;
    Raw8<false> dy = zero8<false>(), zz = zero8<false>();
    auto fetch = [&](int m) {
      dy = fetch8<false, kRagged>(pd, 0, n, m == p.M - 1);
      if (kAct != kActNone) zz = fetch8<false, kRagged>(pz, 0, n, m == p.M - 1);
    };
    if (m0 + warp < m1) fetch(m0 + warp);
    for (int m = m0 + warp; m < m1; m += 8) {
      if (kRagged && n < 8) {
        trim8<false>(dy, pd, 0, n, m == p.M - 1);
        if (kAct != kActNone) trim8<false>(zz, pz, 0, n, m == p.M - 1);
      }
      V8 g = unpack8<false>(dy);
      const V8 z = unpack8<false>(zz);
      pd += 8 * p.lddy;
      if (kAct != kActNone) pz += 8 * p.ldz;
      if (m + 8 < m1) fetch(m + 8);
      if (kAct != kActNone) {
#pragma unroll
        for (int i = 0; i < 8; ++i) g.v[i] *= act_slope(kAct, z.v[i]);
        store8<false, kRagged>(po, c, p.N, g);
        po += 8 * p.lddz;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s.v[i] += g.v[i];
    }
  }
  grid_launch_dependents();
  if (p.part == nullptr) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[warp][lane * 8 + i] = s.v[i];
  __syncthreads();
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col >= p.ldpart) return;  // columns beyond N hold zeros
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) t += sums[w][threadIdx.x];
  p.part[static_cast<size_t>(blockIdx.y) * p.ldpart + col] = t;
}

}  // namespace npd
