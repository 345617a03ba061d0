// The join of a block's branch with the residual stream, and its gradient:
//
//   n[t,c] = x[t,c] r_x[t] (w_post[c] + o)     r_x = 1/sqrt(mean_c x^2 + eps)   (norm of the branch;
//                                              n = x without it)
//   h[t,c] = a residual[t,c] + b gate[.,c] n[t,c]
//   y[t,c] = h[t,c] r_h[t] (w_pre[c] + o)      r_h = 1/sqrt(mean_c h^2 + eps)
//
//   g = dy (w_pre + o),  dh = dh_in + r_h (g - h r_h^2 mean_c(g h)),   dresidual = a dh
//   dn = b gate dh,      dgate = b n dh  (summed over t for a shared gate)
//   v = dn (w_post + o), dx = r_x (v - x r_x^2 mean_c(v x))
//   dw_pre = sum_t dy h r_h,   dw_post = sum_t dn x r_x
//
// Memory bound: every tensor is read once and written once, a row stays in registers between the
// reduction over it and the result.  A CTA works on one row at a time, eight consecutive elements
// per thread and vector, and goes on to row + gridDim; the gains stay in registers and the next
// row's loads are issued before the current row's reductions, so that the memory system has work
// during the barriers.  The sums over rows (gains, shared gate) are kept per thread over all rows
// of the CTA, written once as a partial row per CTA, and added up in a fixed order by a second
// kernel: no atomics, the same bits in every run.
// All arithmetic is fp32; each result is rounded once, when it is stored.  y is taken from the
// fp32 h, not from the rounded h that is stored: one rounding less.
#pragma once

#include "small_kernels.cuh"

namespace npd {

struct NormParams {
  int T, d;
  const __nv_bfloat16* x;     // [T, ldx] or NULL
  const void* residual;       // stream type [T, ldr] or NULL
  const __nv_bfloat16* gate;  // [T, ldg], or one row when ldg == 0, or NULL
  const void* w_post;         // [d] or NULL (gain 1)
  const void* w_pre;          // [d] or NULL (gain 1)
  int post;                   // norm of the branch
  int w_f32;                  // gains are fp32 (else bf16)
  long long ldx, ldr, ldg;
  float eps, offset, res_scale, branch_scale;
  // forward
  void* h;                    // stream type or NULL
  __nv_bfloat16* y;           // or NULL
  long long ldh, ldy;
  // backward (h above is an input there)
  const __nv_bfloat16* dy;    // or NULL
  const void* dh;             // stream type or NULL
  __nv_bfloat16* dx;          // or NULL
  void* dres;                 // stream type or NULL
  __nv_bfloat16* dgate;       // per-token gate gradient, or NULL
  long long lddy, lddh, lddx, lddres, lddgate;
  float* part;                // [gridDim][3][d] partial sums over rows: w_pre, w_post, shared gate
  int want;                   // bit 0: w_pre, bit 1: w_post, bit 2: shared gate
};

namespace norm_cfg {
constexpr int kMaxD = 16384;
// A row takes at most 512 threads (128 registers each).  Up to d = 4096 that is one vector of eight
// per thread, with gains, sums over rows and the next row's loads in registers; beyond, two or four
// vectors per thread, gains re-read (they sit in L1/L2), the sums in shared memory and no prefetch: the
// data of two vectors alone fill the registers, and a row is then long enough to cover its latency.
constexpr int kMaxSmallD = 4096;
constexpr int kMaxThreads = 512;
}  // namespace norm_cfg

// ---- eight consecutive elements ----
struct V8 {
  float v[8];
};
template <bool kF32>
struct Raw8 {
  uint4 q[kF32 ? 2 : 1];
};
// Loads elements [c, c+8) of a row, those below d; the others read as 0.  Rows start on 16-byte
// boundaries and strides are multiples of 16 bytes, so whole vectors are aligned; the last, partial one
// is fetched element by element (nothing past the row's end is read).
template <bool kF32>
__device__ __forceinline__ Raw8<kF32> load8(const void* row, int c, int d) {
  Raw8<kF32> r;
  if (c + 8 <= d) {
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const char*>(row) + static_cast<size_t>(c) * (kF32 ? 4 : 2));
    r.q[0] = *p;
    if (kF32) r.q[kF32 ? 1 : 0] = p[1];
    return r;
  }
  uint32_t w[kF32 ? 8 : 4];
#pragma unroll
  for (int i = 0; i < (kF32 ? 8 : 4); ++i) {
    if (kF32) {
      w[i] = c + i < d ? static_cast<const uint32_t*>(row)[c + i] : 0u;
    } else {
      const uint16_t* e = static_cast<const uint16_t*>(row);
      const uint32_t lo = c + 2 * i < d ? e[c + 2 * i] : 0u, hi = c + 2 * i + 1 < d ? e[c + 2 * i + 1] : 0u;
      w[i] = lo | (hi << 16);
    }
  }
  r.q[0] = make_uint4(w[0], w[1], w[2], w[3]);
  if (kF32) r.q[kF32 ? 1 : 0] = make_uint4(w[kF32 ? 4 : 0], w[kF32 ? 5 : 0], w[kF32 ? 6 : 0], w[kF32 ? 7 : 0]);
  return r;
}
template <bool kF32>
__device__ __forceinline__ Raw8<kF32> zero8() {
  Raw8<kF32> r;
  r.q[0] = make_uint4(0u, 0u, 0u, 0u);
  if (kF32) r.q[kF32 ? 1 : 0] = r.q[0];
  return r;
}
template <bool kF32>
__device__ __forceinline__ V8 unpack8(const Raw8<kF32>& r) {
  V8 o;
  if (kF32) {
    const uint4 a = r.q[0], b = r.q[kF32 ? 1 : 0];
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = __uint_as_float(w[i]);
  } else {
    const uint32_t w[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o.v[2 * i] = bf16_lo(w[i]);
      o.v[2 * i + 1] = bf16_hi(w[i]);
    }
  }
  return o;
}
template <bool kF32>
__device__ __forceinline__ void store8(void* row, int c, int d, const V8& a) {
  if (kF32) {
    float* p = static_cast<float*>(row) + c;
    if (c + 8 <= d) {
      reinterpret_cast<float4*>(p)[0] = make_float4(a.v[0], a.v[1], a.v[2], a.v[3]);
      reinterpret_cast<float4*>(p)[1] = make_float4(a.v[4], a.v[5], a.v[6], a.v[7]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < d) p[i] = a.v[i];
    }
  } else {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(row) + c;
    if (c + 8 <= d) {
      *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(a.v[0], a.v[1]), pack_bf16x2(a.v[2], a.v[3]),
                                                pack_bf16x2(a.v[4], a.v[5]), pack_bf16x2(a.v[6], a.v[7]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < d) p[i] = __float2bfloat16_rn(a.v[i]);
    }
  }
}
// Gains w[c..c+8) + offset (0 beyond d; 1 without a gain).
__device__ __forceinline__ V8 gain8(const void* w, int w_f32, float offset, int c, int d) {
  V8 o;
  if (w == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = 1.f;
    return o;
  }
  // the gains need not be 16-byte aligned: a parameter may be a slice of a larger one
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v = 0.f;
    if (c + i < d)
      v = (w_f32 ? static_cast<const float*>(w)[c + i] : __bfloat162float(static_cast<const __nv_bfloat16*>(w)[c + i])) + offset;
    o.v[i] = v;
  }
  return o;
}

// Sums of N values over the block, the same in every thread.  One barrier; the caller alternates
// `buf` so that a second call may write while slow threads still read the first one's numbers.
template <int N>
__device__ __forceinline__ void block_sum(float (&s)[N], float (*buf)[N]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int k = 0; k < N; ++k) s[k] = warp_sum(s[k]);
  if (warps == 1) return;
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) buf[warp][k] = s[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) s[k] = warp_sum(lane < warps ? buf[lane][k] : 0.f);
}

// Forward.  kVec vectors of eight per thread; vector j of a thread starts at 8 * (threadIdx + j * blockDim).
template <bool kF32, int kVec>
__global__ void __launch_bounds__(norm_cfg::kMaxThreads) norm_fwd_kernel(const NormParams p) {
  __shared__ float red[4][32][1];
  constexpr bool kHold = kVec == 1;  // gains held in registers
  const int nt = blockDim.x;
  const float inv_d = 1.f / static_cast<float>(p.d);
  V8 wp[kVec], wq[kVec], gs[kVec];
  const bool shared_gate = p.gate != nullptr && p.ldg == 0;
  grid_dependency_wait();
  grid_launch_dependents();
  if (kHold) {
    const int c = 8 * threadIdx.x;
    wp[0] = gain8(p.w_post, p.w_f32, p.offset, c, p.d);
    wq[0] = gain8(p.w_pre, p.w_f32, p.offset, c, p.d);
    if (shared_gate) gs[0] = unpack8<false>(load8<false>(p.gate, c, p.d));
  }
  struct Row {
    Raw8<false> x[kVec], g[kVec];
    Raw8<kF32> r[kVec];
  };
  auto fetch = [&](int t) {
    Row o;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt);
      o.x[j] = p.x != nullptr ? load8<false>(p.x + static_cast<size_t>(t) * p.ldx, c, p.d) : zero8<false>();
      o.r[j] = p.residual != nullptr
                  ? load8<kF32>(static_cast<const char*>(p.residual) + static_cast<size_t>(t) * p.ldr * (kF32 ? 4 : 2), c, p.d)
                  : zero8<kF32>();
      if (p.gate != nullptr && !shared_gate) o.g[j] = load8<false>(p.gate + static_cast<size_t>(t) * p.ldg, c, p.d);
    }
    return o;
  };
  int t = blockIdx.x, par = 0;
  Row next;
  if (kHold && t < p.T) next = fetch(t);
  for (; t < p.T; t += gridDim.x, par ^= 1) {
    const Row cur = kHold ? next : fetch(t);
    if (kHold && t + static_cast<int>(gridDim.x) < p.T) next = fetch(t + gridDim.x);
    V8 r[kVec];
    float scale = p.branch_scale;
    if (p.post) {
      float s[1] = {0.f};
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const V8 x = unpack8<false>(cur.x[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] = fmaf(x.v[i], x.v[i], s[0]);
      }
      block_sum<1>(s, red[2 * par]);
      scale *= rsqrtf(fmaf(s[0], inv_d, p.eps));
    }
    float s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt);
      if (!kHold) {
        if (p.post) wp[j] = gain8(p.w_post, p.w_f32, p.offset, c, p.d);
        if (shared_gate) gs[j] = unpack8<false>(load8<false>(p.gate, c, p.d));
      }
      const V8 x = unpack8<false>(cur.x[j]);
      r[j] = unpack8<kF32>(cur.r[j]);
      V8 g;
      if (p.gate != nullptr) g = shared_gate ? gs[j] : unpack8<false>(cur.g[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float b = x.v[i] * scale;
        if (p.post) b *= wp[j].v[i];
        if (p.gate != nullptr) b *= g.v[i];
        const float h = fmaf(p.res_scale, r[j].v[i], b);
        r[j].v[i] = h;
        s[0] = fmaf(h, h, s[0]);
      }
      if (p.h != nullptr)
        store8<kF32>(static_cast<char*>(p.h) + static_cast<size_t>(t) * p.ldh * (kF32 ? 4 : 2), c, p.d, r[j]);
    }
    if (p.y == nullptr) continue;
    block_sum<1>(s, red[2 * par + 1]);
    const float rh = rsqrtf(fmaf(s[0], inv_d, p.eps));
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt);
      if (!kHold) wq[j] = gain8(p.w_pre, p.w_f32, p.offset, c, p.d);
      V8 o;
#pragma unroll
      for (int i = 0; i < 8; ++i) o.v[i] = r[j].v[i] * rh * wq[j].v[i];
      store8<false>(p.y + static_cast<size_t>(t) * p.ldy, c, p.d, o);
    }
  }
}

// Backward.  The sums over rows live in registers (kVec == 1) or in shared memory (dynamic, [3][d]).
template <bool kF32, int kVec>
__global__ void __launch_bounds__(norm_cfg::kMaxThreads) norm_bwd_kernel(const NormParams p) {
  __shared__ float red3[2][32][3];
  __shared__ float red1[2][32][1];
  extern __shared__ float acc_smem[];
  constexpr bool kHold = kVec == 1;
  const int nt = blockDim.x;
  const float inv_d = 1.f / static_cast<float>(p.d);
  const bool shared_gate = p.gate != nullptr && p.ldg == 0, token_gate = p.gate != nullptr && p.ldg != 0;
  V8 wp[kVec], wq[kVec], gs[kVec];
  V8 acc[3];  // kHold: sums over this CTA's rows of dy h r_h, dn x r_x, b n dh
  if (kHold) {
    const int c = 8 * threadIdx.x;
    grid_dependency_wait();
    wp[0] = gain8(p.w_post, p.w_f32, p.offset, c, p.d);
    wq[0] = gain8(p.w_pre, p.w_f32, p.offset, c, p.d);
    if (shared_gate) gs[0] = unpack8<false>(load8<false>(p.gate, c, p.d));
#pragma unroll
    for (int a = 0; a < 3; ++a)
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[a].v[i] = 0.f;
  } else {
    // every thread clears, adds to and reads back its own columns only: no barrier needed
    for (int a = 0; a < 3; ++a)
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        for (int i = 0; i < 8; ++i) {
          const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt) + i;
          if (c < p.d) acc_smem[a * p.d + c] = 0.f;
        }
    grid_dependency_wait();
  }
  struct Row {
    Raw8<false> dy[kVec], x[kVec], g[kVec];
    Raw8<kF32> h[kVec], dh[kVec];
  };
  const size_t es = kF32 ? 4 : 2;
  auto fetch = [&](int t) {
    Row o;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt);
      if (p.dy != nullptr) {
        o.dy[j] = load8<false>(p.dy + static_cast<size_t>(t) * p.lddy, c, p.d);
        o.h[j] = load8<kF32>(static_cast<const char*>(p.h) + static_cast<size_t>(t) * p.ldh * es, c, p.d);
      } else {
        o.dy[j] = zero8<false>();
        o.h[j] = zero8<kF32>();
      }
      o.dh[j] = p.dh != nullptr ? load8<kF32>(static_cast<const char*>(p.dh) + static_cast<size_t>(t) * p.lddh * es, c, p.d)
                                : zero8<kF32>();
      o.x[j] = p.x != nullptr ? load8<false>(p.x + static_cast<size_t>(t) * p.ldx, c, p.d) : zero8<false>();
      if (token_gate) o.g[j] = load8<false>(p.gate + static_cast<size_t>(t) * p.ldg, c, p.d);
    }
    return o;
  };
  int t = blockIdx.x, par = 0;
  Row next;
  if (kHold && t < p.T) next = fetch(t);
  for (; t < p.T; t += gridDim.x, par ^= 1) {
    const Row cur = kHold ? next : fetch(t);
    if (kHold && t + static_cast<int>(gridDim.x) < p.T) next = fetch(t + gridDim.x);
    V8 vv[kVec];
    float s[3] = {0.f, 0.f, 0.f};  // sum h^2, sum g h, sum x^2
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt);
      if (!kHold) wq[j] = gain8(p.w_pre, p.w_f32, p.offset, c, p.d);
      const V8 dy = unpack8<false>(cur.dy[j]), h = unpack8<kF32>(cur.h[j]), x = unpack8<false>(cur.x[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[0] = fmaf(h.v[i], h.v[i], s[0]);
        s[1] = fmaf(dy.v[i] * wq[j].v[i], h.v[i], s[1]);
        s[2] = fmaf(x.v[i], x.v[i], s[2]);
      }
    }
    block_sum<3>(s, red3[par]);
    const float rh = p.dy != nullptr ? rsqrtf(fmaf(s[0], inv_d, p.eps)) : 0.f;
    const float ch = rh * rh * s[1] * inv_d;
    const float rx = p.post ? rsqrtf(fmaf(s[2], inv_d, p.eps)) : 1.f;
    float q[1] = {0.f};  // sum v x
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt);
      if (!kHold) {
        wq[j] = gain8(p.w_pre, p.w_f32, p.offset, c, p.d);
        wp[j] = gain8(p.w_post, p.w_f32, p.offset, c, p.d);
        if (shared_gate) gs[j] = unpack8<false>(load8<false>(p.gate, c, p.d));
      }
      const V8 dy = unpack8<false>(cur.dy[j]), h = unpack8<kF32>(cur.h[j]), x = unpack8<false>(cur.x[j]),
               dh = unpack8<kF32>(cur.dh[j]);
      V8 o, dg, g;
      if (p.gate != nullptr) g = shared_gate ? gs[j] : unpack8<false>(cur.g[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float hi = h.v[i], xi = x.v[i];
        const float a0 = dy.v[i] * hi * rh;
        const float dhi = fmaf(rh, fmaf(dy.v[i], wq[j].v[i], -hi * ch), dh.v[i]);
        o.v[i] = p.res_scale * dhi;
        const float xn = xi * rx;                                   // x, normalised if there is a norm
        const float n = p.post ? xn * wp[j].v[i] : xn;
        const float bd = p.branch_scale * dhi;
        dg.v[i] = bd * n;
        const float dn = p.gate == nullptr ? bd : bd * g.v[i];
        const float a1 = dn * xn;
        const float v = p.post ? dn * wp[j].v[i] : dn;
        q[0] = fmaf(v, xi, q[0]);
        vv[j].v[i] = v;
        if (kHold) {
          acc[0].v[i] += a0;
          acc[1].v[i] += a1;
          acc[2].v[i] += dg.v[i];
        } else if (c + i < p.d) {
          acc_smem[c + i] += a0;
          acc_smem[p.d + c + i] += a1;
          acc_smem[2 * p.d + c + i] += dg.v[i];
        }
      }
      if (p.dres != nullptr)
        store8<kF32>(static_cast<char*>(p.dres) + static_cast<size_t>(t) * p.lddres * es, c, p.d, o);
      if (p.dgate != nullptr) store8<false>(p.dgate + static_cast<size_t>(t) * p.lddgate, c, p.d, dg);
    }
    if (p.dx == nullptr) continue;
    float cx = 0.f;
    if (p.post) {
      block_sum<1>(q, red1[par]);
      cx = rx * rx * q[0] * inv_d;
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt);
      const V8 x = unpack8<false>(cur.x[j]);
      V8 o;
#pragma unroll
      for (int i = 0; i < 8; ++i) o.v[i] = rx * fmaf(-x.v[i], cx, vv[j].v[i]);
      store8<false>(p.dx + static_cast<size_t>(t) * p.lddx, c, p.d, o);
    }
  }
  grid_launch_dependents();
  if (p.want == 0) return;
  float* part = p.part + static_cast<size_t>(blockIdx.x) * 3 * p.d;
#pragma unroll
  for (int a = 0; a < 3; ++a) {
    if (((p.want >> a) & 1) == 0) continue;
    if (kHold) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = 8 * threadIdx.x + i;
        if (c < p.d) part[static_cast<size_t>(a) * p.d + c] = acc[a].v[i];
      }
    } else {
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        for (int i = 0; i < 8; ++i) {
          const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt) + i;
          if (c < p.d) part[static_cast<size_t>(a) * p.d + c] = acc_smem[a * p.d + c];
        }
    }
  }
}

// out_a[c] = sum over `rows` partial rows, in a fixed order: 16 interleaved runs, then the runs.
__global__ void __launch_bounds__(512) column_sum_kernel(const float* __restrict__ part, int rows, long long row_stride,
                                                        long long array_stride, int d, float* out0, float* out1,
                                                        float* out2) {
  __shared__ float s[16][33];
  float* out = blockIdx.y == 0 ? out0 : (blockIdx.y == 1 ? out1 : out2);
  const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  grid_dependency_wait();
  grid_launch_dependents();
  if (out == nullptr) return;
  float v = 0.f;
  if (c < d) {
    const float* q = part + blockIdx.y * array_stride + c;
#pragma unroll 4
    for (int r = run; r < rows; r += 16) v += q[static_cast<size_t>(r) * row_stride];
  }
  s[run][lane] = v;
  __syncthreads();
  if (run == 0 && c < d) {
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) t += s[k][lane];
    out[c] = t;
  }
}

}  // namespace npd
