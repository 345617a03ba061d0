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
// per thread and vector, and goes on to row + gridDim; gains stay in registers as far as they fit, and
// the next rows' loads are under way during the current row's reductions (the forward holds them in registers, the
// backward with a bf16 stream in a ring in shared memory).  The sums over rows (gains, shared gate) are kept per thread over all rows
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
  float* part;                // [gridDim][2][part_d] partial sums over rows: of dy h r_h, and S (see norm_bwd_kernel)
  int part_d;                 // d rounded up to a multiple of 4
  int want;                   // bit 0: w_pre, bit 1: w_post, bit 2: shared gate
};

namespace norm_cfg {
constexpr int kMaxD = 16384;
// One vector of eight per thread, gains (and sums over rows) in registers, up to d = 8192 (1024 threads of 64
// registers) in the forward and 4096 (512 threads of 128) in the backward; beyond, two or four vectors per thread
// (at most 512 of them), gains re-read (they sit in L1/L2), sums over rows in shared memory.
constexpr int kMaxSmallFwd = 8192, kMaxSmallBwd = 4096;
constexpr int kMaxSmem = 2 * kMaxD * 4;  // dynamic shared memory a launch may ask for: sums over the widest row
constexpr int kRing = 2;  // rows in flight per CTA of the backward
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
// Gains w[c..c+8) + offset (0 beyond d; 1 without a gain).  kWide: with 16-byte loads where the address allows it,
// for the kernels that read their gains again for every row.
template <bool kWide>
__device__ __forceinline__ V8 gain8(const void* w, int w_f32, float offset, int c, int d) {
  V8 o;
  if (w == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = 1.f;
    return o;
  }
  // the gains need not be 16-byte aligned: a parameter may be a slice of a larger one
  if (kWide && (reinterpret_cast<uintptr_t>(w) & 15u) == 0 && c + 8 <= d) {
    o = w_f32 ? unpack8<true>(load8<true>(w, c, d)) : unpack8<false>(load8<false>(w, c, d));
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] += offset;
    return o;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v = 0.f;
    if (c + i < d)
      v = (w_f32 ? static_cast<const float*>(w)[c + i] : __bfloat162float(static_cast<const __nv_bfloat16*>(w)[c + i])) + offset;
    o.v[i] = v;
  }
  return o;
}

// ---- the same as four pairs for the packed fp32 instructions (two results per instruction and thread: with
// scalar ones these kernels are bound by the instructions they issue, not by memory) ----
struct P8 {
  unsigned long long p[4];
};
__device__ __forceinline__ unsigned long long pair2(float lo, float hi) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 unpair2(unsigned long long a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a));
  return r;
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float sum2(unsigned long long a) {
  const float2 v = unpair2(a);
  return v.x + v.y;
}
__device__ __forceinline__ P8 pack8(const V8& a) {
  P8 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o.p[i] = pair2(a.v[2 * i], a.v[2 * i + 1]);
  return o;
}
template <bool kF32>
__device__ __forceinline__ P8 pairs8(const Raw8<kF32>& r) {
  return pack8(unpack8<kF32>(r));
}
template <bool kF32>
__device__ __forceinline__ void store8(void* row, int c, int d, const P8& a) {
  V8 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 q = unpair2(a.p[i]);
    v.v[2 * i] = q.x;
    v.v[2 * i + 1] = q.y;
  }
  store8<kF32>(row, c, d, v);
}

// ---- a ring of rows in shared memory, filled by asynchronous copies; slot s of a stage holds 16 bytes of every
// thread, and every thread copies and reads only its own, so the ring needs no barrier ----
__device__ __forceinline__ void async_copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Waits until at most kPending of this thread's newest groups are in flight.
template <int kPending>
__device__ __forceinline__ void async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory");
}
__device__ __forceinline__ uint4 ring_get(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

// Sums of N values over the block, the same in every thread, in a fixed order.  One barrier; the caller
// alternates `buf` so that a second call may write while slow threads still read the first one's numbers.
// The places of warps that do not exist hold zeros.
template <int N>
struct SumBuf {
  float4 v[N][8];
};
template <int N>
__device__ __forceinline__ void clear_sums(SumBuf<N>* buf, int count) {
  float* f = reinterpret_cast<float*>(buf);
  for (int i = threadIdx.x; i < count * N * 32; i += blockDim.x) f[i] = 0.f;
}
// kWide: the block may have more than 16 warps.
template <int N, bool kWide = false>
__device__ __forceinline__ void block_sum(float (&s)[N], SumBuf<N>& buf) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int k = 0; k < N; ++k) s[k] = warp_sum(s[k]);
  if (warps == 1) return;
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) reinterpret_cast<float*>(&buf.v[k][0])[warp] = s[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float4 a = buf.v[k][0], b = buf.v[k][1];
    s[k] = ((a.x + a.y) + (a.z + a.w)) + ((b.x + b.y) + (b.z + b.w));
    if (warps > 8) {
      const float4 c = buf.v[k][2], e = buf.v[k][3];
      s[k] += ((c.x + c.y) + (c.z + c.w)) + ((e.x + e.y) + (e.z + e.w));
    }
    if (kWide && warps > 16) {
      const float4 c = buf.v[k][4], e = buf.v[k][5], f = buf.v[k][6], g = buf.v[k][7];
      s[k] += (((c.x + c.y) + (c.z + c.w)) + ((e.x + e.y) + (e.z + e.w))) + (((f.x + f.y) + (f.z + f.w)) + ((g.x + g.y) + (g.z + g.w)));
    }
  }
}

// What is missing in a call costs no branches in the arithmetic: a missing gain or gate is a gain of 1, a
// missing operand zeros, and a branch without a norm has r_x = 1.

// Forward.  kVec vectors of eight per thread; vector j of a thread starts at 8 * (threadIdx + j * blockDim).
template <bool kF32, int kVec, int kThreads>
__global__ void __launch_bounds__(kThreads, kVec == 1 ? 1024 / kThreads : 1) norm_fwd_kernel(const NormParams p) {
  __shared__ SumBuf<1> red[4];
  constexpr bool kHold = kVec == 1;  // gains held in registers, the next row's loads in flight
  constexpr size_t es = kF32 ? 4 : 2;
  const int nt = blockDim.x;
  const float inv_d = 1.f / static_cast<float>(p.d);
  const bool token_gate = p.gate != nullptr && p.ldg != 0;
  P8 wp[kVec], wq[kVec];  // gain of the branch times a shared gate; gain of y
  grid_dependency_wait();
  grid_launch_dependents();
  auto gains = [&](int j) {
    const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt);
    V8 w = gain8<!kHold>(p.w_post, p.w_f32, p.offset, c, p.d);
    if (p.gate != nullptr && !token_gate) {
      const V8 g = unpack8<false>(load8<false>(p.gate, c, p.d));
#pragma unroll
      for (int i = 0; i < 8; ++i) w.v[i] *= g.v[i];
    }
    wp[j] = pack8(w);
    wq[j] = pack8(gain8<!kHold>(p.w_pre, p.w_f32, p.offset, c, p.d));
  };
  if (kHold) gains(0);
  clear_sums(red, 4);
  __syncthreads();
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
                  ? load8<kF32>(static_cast<const char*>(p.residual) + static_cast<size_t>(t) * p.ldr * es, c, p.d)
                  : zero8<kF32>();
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
    float scale = p.branch_scale;
    if (p.post) {
      unsigned long long q = 0ull;
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const P8 x = pairs8<false>(cur.x[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) q = fma2(x.p[i], x.p[i], q);
      }
      float s[1] = {sum2(q)};
      block_sum<1, (kThreads > 512)>(s, red[2 * par]);
      scale *= rsqrtf(fmaf(s[0], inv_d, p.eps));
    }
    const unsigned long long scale2 = pair2(scale, scale), res2 = pair2(p.res_scale, p.res_scale);
    unsigned long long q = 0ull;
    P8 h[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt);
      if (!kHold) gains(j);
      const P8 x = pairs8<false>(cur.x[j]), r = pairs8<kF32>(cur.r[j]);
      P8 w = wp[j];
      if (token_gate) {
        const P8 g = pairs8<false>(cur.g[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) w.p[i] = mul2(w.p[i], g.p[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned long long b = mul2(mul2(x.p[i], scale2), w.p[i]);
        h[j].p[i] = fma2(res2, r.p[i], b);
        q = fma2(h[j].p[i], h[j].p[i], q);
      }
      if (p.h != nullptr) store8<kF32>(static_cast<char*>(p.h) + static_cast<size_t>(t) * p.ldh * es, c, p.d, h[j]);
    }
    if (p.y == nullptr) continue;
    float s[1] = {sum2(q)};
    block_sum<1, (kThreads > 512)>(s, red[2 * par + 1]);
    const float rh = rsqrtf(fmaf(s[0], inv_d, p.eps));
    const unsigned long long rh2 = pair2(rh, rh);
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt);
      P8 o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o.p[i] = mul2(mul2(h[j].p[i], rh2), wq[j].p[i]);
      store8<false>(p.y + static_cast<size_t>(t) * p.ldy, c, p.d, o);
    }
  }
}

// Backward.  With G = b gate gain_post, v = dh G, and the sums over rows behind the gains and a shared gate are
// d_post = b gate S and d_gate = b gain_post S with the same S = sum_t dh x r_x (times the row's gate, if
// every token has its own), so a column needs two sums and two gains: they stay in registers with kVec == 1
// (80 registers, four CTAs of 192 threads per SM at d = 1536: enough warps to cover each other's reductions
// and loads; with prefetched rows as well, three warps per scheduler waited for their own shuffles, and with
// gains in shared memory that memory's pipe was the limit).  Otherwise the sums are in shared memory
// (dynamic, [2][d]) and gains are re-read.
// kForm > 0: every operand and result exists, no per-token gate, d a multiple of 8 (no vector is partly outside the
// row); 2: of 256 (no thread is outside it): the same arithmetic without the tests for it (d = 1536 with form 1:
// 230 us instead of 198 at T = 65,536; d = 1000 with form 0: 78 us instead of 50 at T = 16,384).  With a bf16 stream rows then arrive
// through a ring of kRing stages in shared memory (asynchronous copies, two rows ahead), so that loads are in
// flight during the reductions without taking registers: T = 65,536, d = 1536 takes 198 us with it and 259 us
// without.  With an fp32 stream the ring is slower (387 us against 315 us).
template <bool kF32, int kVec, int kForm, int kThreads, int kBlocks>
__global__ void __launch_bounds__(kThreads, kBlocks) norm_bwd_kernel(const NormParams p) {
  __shared__ SumBuf<3> red3[2];
  __shared__ SumBuf<1> red1[2];
  extern __shared__ __align__(16) float dyn[];  // sums over rows, or the ring
  constexpr bool kHold = kVec == 1, kFull = kForm > 0;
  constexpr int kRing = norm_cfg::kRing;
  constexpr bool kRows = kFull && !kF32;  // rows arrive through the ring
  constexpr size_t es = kF32 ? 4 : 2;
  const int nt = blockDim.x;
  const float inv_d = 1.f / static_cast<float>(p.d);
  const bool shared_gate = p.gate != nullptr && p.ldg == 0, token_gate = !kFull && p.gate != nullptr && p.ldg != 0;
  const bool have_y = kFull || p.dy != nullptr, have_dh = kFull || p.dh != nullptr, have_x = kFull || p.x != nullptr;
  P8 acc[2];  // kHold: sums over this CTA's rows of dy h r_h and of dh x r_x
  P8 held[2];  // kHold: gain of y, G
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[0].p[i] = acc[1].p[i] = held[0].p[i] = held[1].p[i] = 0ull;
  auto shared_gate8 = [&](int c) { return shared_gate ? unpack8<false>(load8<false>(p.gate, c, p.d)) : gain8<!kHold>(nullptr, 0, 0.f, c, p.d); };
  // which: 0 = gain of y, 1 = G (without a per-token gate)
  auto read_gain = [&](int which, int c) {
    if (which == 0) return pack8(gain8<!kHold>(p.w_pre, p.w_f32, p.offset, c, p.d));
    V8 w = gain8<!kHold>(p.w_post, p.w_f32, p.offset, c, p.d);
    const V8 g = shared_gate8(c);
#pragma unroll
    for (int i = 0; i < 8; ++i) w.v[i] *= p.branch_scale * g.v[i];
    return pack8(w);
  };
  // !kHold: the sums, [sum][vector][half] planes of 16 bytes per thread
  ulonglong2* sums = reinterpret_cast<ulonglong2*>(dyn);
  auto gain = [&](int which, int j) {
    return kHold ? held[which] : read_gain(which, 8 * (static_cast<int>(threadIdx.x) + j * nt));
  };
  clear_sums(red3, 2);
  clear_sums(red1, 2);
  grid_dependency_wait();
  if (kHold) {
    held[0] = read_gain(0, 8 * static_cast<int>(threadIdx.x));
    held[1] = read_gain(1, 8 * static_cast<int>(threadIdx.x));
  } else {
    // every thread clears, adds to and reads back its own columns only: no barrier needed
    for (int i = 0; i < 4 * kVec; ++i) sums[i * nt + threadIdx.x] = make_ulonglong2(0ull, 0ull);
  }
  __syncthreads();
  struct Row {
    Raw8<false> dy[kVec], x[kVec], g[kVec];
    Raw8<kF32> h[kVec], dh[kVec];
  };
  const int d_ = kFull ? 1 << 30 : p.d;  // kFull: no vector reaches past the row ...
  const bool active = kForm != 1 || 8 * static_cast<int>(threadIdx.x) < p.d;  // ... and threads beyond it hold zeros
  auto fetch = [&](int t) {
    Row o;
    if (!active) {
      o.dy[0] = o.x[0] = zero8<false>();
      o.h[0] = o.dh[0] = zero8<kF32>();
      return o;
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt);
      if (have_y) {
        o.dy[j] = load8<false>(p.dy + static_cast<size_t>(t) * p.lddy, c, d_);
        o.h[j] = load8<kF32>(static_cast<const char*>(p.h) + static_cast<size_t>(t) * p.ldh * es, c, d_);
      } else {
        o.dy[j] = zero8<false>();
        o.h[j] = zero8<kF32>();
      }
      o.dh[j] = have_dh ? load8<kF32>(static_cast<const char*>(p.dh) + static_cast<size_t>(t) * p.lddh * es, c, d_) : zero8<kF32>();
      o.x[j] = have_x ? load8<false>(p.x + static_cast<size_t>(t) * p.ldx, c, d_) : zero8<false>();
      if (token_gate) o.g[j] = load8<false>(p.gate + static_cast<size_t>(t) * p.ldg, c, d_);
    }
    return o;
  };
  // the ring: slots of a stage are dy, x, h, dh
  constexpr int kSlots = 4;
  const uint32_t slot = 16u * static_cast<uint32_t>(nt), ring0 = smem_u32(dyn) + 16u * threadIdx.x;
  auto issue = [&](int t, int stage) {
    if (t < p.T && active) {
      const uint32_t at = ring0 + static_cast<uint32_t>(stage) * kSlots * slot;
      async_copy16(at, p.dy + static_cast<size_t>(t) * p.lddy + 8 * threadIdx.x);
      async_copy16(at + slot, p.x + static_cast<size_t>(t) * p.ldx + 8 * threadIdx.x);
      async_copy16(at + 2 * slot, static_cast<const __nv_bfloat16*>(p.h) + static_cast<size_t>(t) * p.ldh + 8 * threadIdx.x);
      async_copy16(at + 3 * slot, static_cast<const __nv_bfloat16*>(p.dh) + static_cast<size_t>(t) * p.lddh + 8 * threadIdx.x);
    }
    async_commit();
  };
  auto take = [&](int stage) {
    Row o;
    if (!active) {
      o.dy[0].q[0] = o.x[0].q[0] = o.h[0].q[0] = o.dh[0].q[0] = make_uint4(0u, 0u, 0u, 0u);
      return o;
    }
    const uint32_t at = ring0 + static_cast<uint32_t>(stage) * kSlots * slot;
    o.dy[0].q[0] = ring_get(at);
    o.x[0].q[0] = ring_get(at + slot);
    o.h[0].q[0] = ring_get(at + 2 * slot);
    o.dh[0].q[0] = ring_get(at + 3 * slot);
    return o;
  };
  const unsigned long long rs2 = pair2(p.res_scale, p.res_scale);
  int par = 0, stage = 0;
  if (kRows)
    for (int i = 0; i < kRing; ++i) issue(blockIdx.x + i * static_cast<int>(gridDim.x), i);
  for (int t = blockIdx.x; t < p.T; t += gridDim.x, par ^= 1) {
    Row cur;
    if (kRows) {
      async_wait<kRing - 1>();
      cur = take(stage);
    } else {
      cur = fetch(t);
    }
    P8 vv[kVec];
    unsigned long long s0 = 0ull, s1 = 0ull, s2 = 0ull;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const P8 dy = pairs8<false>(cur.dy[j]), h = pairs8<kF32>(cur.h[j]), x = pairs8<false>(cur.x[j]), wq = gain(0, j);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s0 = fma2(h.p[i], h.p[i], s0);
        s1 = fma2(mul2(dy.p[i], wq.p[i]), h.p[i], s1);
        s2 = fma2(x.p[i], x.p[i], s2);
      }
    }
    if (kRows) {
      // the stage's values are in registers: its place is free for the row kRing further on
      issue(t + kRing * static_cast<int>(gridDim.x), stage);
      stage = stage + 1 == kRing ? 0 : stage + 1;
    }
    float s[3] = {sum2(s0), sum2(s1), sum2(s2)};  // sum h^2, sum g h, sum x^2
    block_sum<3>(s, red3[par]);
    const float rh = have_y ? rsqrtf(fmaf(s[0], inv_d, p.eps)) : 0.f;
    const float rx = p.post ? rsqrtf(fmaf(s[2], inv_d, p.eps)) : 1.f;
    const float ch = -rh * rh * s[1] * inv_d;
    const unsigned long long rh2 = pair2(rh, rh), ch2 = pair2(ch, ch), rx2 = pair2(rx, rx);
    unsigned long long q = 0ull;  // sum v x
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt);
      const P8 dy = pairs8<false>(cur.dy[j]), h = pairs8<kF32>(cur.h[j]), x = pairs8<false>(cur.x[j]),
               dh = pairs8<kF32>(cur.dh[j]);
      const P8 wq = gain(0, j), G = gain(1, j);
      P8 o, dg, g, a0, a1, d2s;
      if (token_gate) g = pairs8<false>(cur.g[j]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned long long d2 = fma2(rh2, fma2(h.p[i], ch2, mul2(dy.p[i], wq.p[i])), dh.p[i]);  // dh
        o.p[i] = mul2(rs2, d2);
        unsigned long long xn = mul2(x.p[i], rx2);  // x, normalised if there is a norm
        unsigned long long v = mul2(d2, G.p[i]);
        if (token_gate) {
          dg.p[i] = mul2(v, xn);
          v = mul2(v, g.p[i]);
          xn = mul2(xn, g.p[i]);
        }
        q = fma2(v, x.p[i], q);
        vv[j].p[i] = v;
        if (kHold) {
          acc[0].p[i] = fma2(mul2(dy.p[i], h.p[i]), rh2, acc[0].p[i]);
          acc[1].p[i] = fma2(d2, xn, acc[1].p[i]);
        } else {
          a0.p[i] = mul2(dy.p[i], h.p[i]);
          a1.p[i] = xn;
          d2s.p[i] = d2;
        }
      }
      if (!kHold) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          ulonglong2* u = sums + (2 * j + half) * nt + threadIdx.x;
          ulonglong2* w = sums + (2 * (kVec + j) + half) * nt + threadIdx.x;
          const ulonglong2 su = *u, sw = *w;
          *u = make_ulonglong2(fma2(a0.p[2 * half], rh2, su.x), fma2(a0.p[2 * half + 1], rh2, su.y));
          *w = make_ulonglong2(fma2(d2s.p[2 * half], a1.p[2 * half], sw.x), fma2(d2s.p[2 * half + 1], a1.p[2 * half + 1], sw.y));
        }
      }
      if (kFull ? active : p.dres != nullptr)
        store8<kF32>(static_cast<char*>(p.dres) + static_cast<size_t>(t) * p.lddres * es, c, d_, o);
      if (token_gate && p.dgate != nullptr) store8<false>(p.dgate + static_cast<size_t>(t) * p.lddgate, c, d_, dg);
    }
    if (!kFull && p.dx == nullptr) continue;
    if (p.post) {
      float sq[1] = {sum2(q)};
      block_sum<1>(sq, red1[par]);
      const float cx = -rx * rx * sq[0] * inv_d;
      const unsigned long long cx2 = pair2(cx, cx);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const P8 x = pairs8<false>(cur.x[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) vv[j].p[i] = mul2(rx2, fma2(x.p[i], cx2, vv[j].p[i]));
      }
    }
    if (!active) continue;
#pragma unroll
    for (int j = 0; j < kVec; ++j)
      store8<false>(p.dx + static_cast<size_t>(t) * p.lddx, 8 * (static_cast<int>(threadIdx.x) + j * nt), d_, vv[j]);
  }
  grid_launch_dependents();
  if (p.want == 0) return;
  float* part = p.part + static_cast<size_t>(blockIdx.x) * 2 * p.part_d;
  if (kHold) {
    // rows of part_d floats: 16-byte stores; columns beyond d hold zeros
    const int c = 8 * threadIdx.x;
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int i = 0; i < 4; i += 2)
        if (c + 2 * i < p.part_d)
          *reinterpret_cast<ulonglong2*>(part + static_cast<size_t>(a) * p.part_d + c + 2 * i) = make_ulonglong2(acc[a].p[i], acc[a].p[i + 1]);
  } else {
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        for (int half = 0; half < 2; ++half) {
          const int c = 8 * (static_cast<int>(threadIdx.x) + j * nt) + 4 * half;
          if (c < p.part_d)
            *reinterpret_cast<ulonglong2*>(part + static_cast<size_t>(a) * p.part_d + c) = sums[(2 * (a * kVec + j) + half) * nt + threadIdx.x];
        }
  }
}

// Sums of 32 columns from c0 on over `rows` rows of `part` (row_stride floats apart, a multiple of 4, 16-byte
// aligned, readable up to a multiple of 4 columns), in a fixed order: 128 interleaved runs of four columns per
// thread, all of a thread's loads in flight together, then the runs.  Block of 1024; warp w returns column c0 + w
// in every lane.
__device__ __forceinline__ float column_total(const float* part, int rows, long long row_stride, int c0, int d) {
  __shared__ float s[128][33];
  const int quad = threadIdx.x & 7, run = threadIdx.x >> 3;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c0 + 4 * quad < d) {
    const float* q = part + c0 + 4 * quad;
#pragma unroll 8
    for (int r = run; r < rows; r += 128) {
      const float4 u = *reinterpret_cast<const float4*>(q + static_cast<size_t>(r) * row_stride);
      v.x += u.x;
      v.y += u.y;
      v.z += u.z;
      v.w += u.w;
    }
  }
  s[run][4 * quad] = v.x;
  s[run][4 * quad + 1] = v.y;
  s[run][4 * quad + 2] = v.z;
  s[run][4 * quad + 3] = v.w;
  __syncthreads();
  const int lane = threadIdx.x & 31, col = threadIdx.x >> 5;
  return warp_sum((s[lane][col] + s[lane + 32][col]) + (s[lane + 64][col] + s[lane + 96][col]));
}

// The gradients of the gains and of a shared gate from the partial sums: blockIdx.y 0: d_pre, 1: d_post and d_gate.
__global__ void __launch_bounds__(1024) norm_sums_kernel(const NormParams p, int rows, float* d_pre, float* d_post, float* d_gate) {
  grid_dependency_wait();
  grid_launch_dependents();
  if (blockIdx.y == 0 ? d_pre == nullptr : (d_post == nullptr && d_gate == nullptr)) return;
  const int c0 = blockIdx.x * 32, c = c0 + (static_cast<int>(threadIdx.x) >> 5);
  const float t = column_total(p.part + static_cast<size_t>(blockIdx.y) * p.part_d, rows, 2ll * p.part_d, c0, p.d);
  if ((threadIdx.x & 31) != 0 || c >= p.d) return;
  if (blockIdx.y == 0) {
    d_pre[c] = t;
    return;
  }
  // S -> b gate S and b gain_post S (a per-token gate is already in S)
  const float gate = p.gate != nullptr && p.ldg == 0 ? __bfloat162float(p.gate[c]) : 1.f;
  if (d_post != nullptr) d_post[c] = p.branch_scale * gate * t;
  if (d_gate != nullptr) {
    float w = 1.f;
    if (p.w_post != nullptr)
      w = (p.w_f32 ? static_cast<const float*>(p.w_post)[c] : __bfloat162float(static_cast<const __nv_bfloat16*>(p.w_post)[c])) + p.offset;
    d_gate[c] = p.branch_scale * w * t;
  }
}

// out[c] = sum over `rows` partial rows of row_stride (a multiple of 4) floats.
__global__ void __launch_bounds__(1024) column_sum_kernel(const float* __restrict__ part, int rows, long long row_stride, int d, float* out) {
  grid_dependency_wait();
  grid_launch_dependents();
  const int c0 = blockIdx.x * 32, c = c0 + (static_cast<int>(threadIdx.x) >> 5);
  const float t = column_total(part, rows, row_stride, c0, d);
  if ((threadIdx.x & 31) == 0 && c < d) out[c] = t;
}

}  // namespace npd
