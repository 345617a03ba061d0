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
  int span;                   // narrow rows: threads per row (8, 16 or 32)
};

namespace norm_cfg {
constexpr int kMaxD = 16384;
// One vector of eight per thread, gains (and sums over rows) in registers, up to d = 8192 (1024 threads of 64
// registers) in the forward and 4096 (512 threads of 128) in the backward; beyond, two or four vectors per thread
// (at most 512 of them), sums over rows (and up to d = 8192 gains) in shared memory.
constexpr int kMaxSmallFwd = 8192, kMaxSmallBwd = 4096;
constexpr int kMaxSmem = 2 * kMaxD * 4;  // dynamic shared memory a launch may ask for: sums over the widest row
constexpr int kRing = 2;  // rows in flight per CTA of the backward
// Rows of at most 256 elements lie within a warp (8, 16 or 32 threads each): a block of 256 threads takes several
// of them at a time, and none of its reductions needs a barrier.
constexpr int kNarrowD = 256, kNarrowThreads = 256;
}  // namespace norm_cfg

// ---- eight consecutive elements ----
struct V8 {
  float v[8];
};
template <bool kF32>
struct Raw8 {
  uint4 q[kF32 ? 2 : 1];
};
template <bool kF32>
__device__ __forceinline__ Raw8<kF32> zero8() {
  Raw8<kF32> r;
  r.q[0] = make_uint4(0u, 0u, 0u, 0u);
  if (kF32) r.q[kF32 ? 1 : 0] = r.q[0];
  return r;
}
// Loads elements [c, c+8) of a row, those below d; the others read as 0.  Rows start on 16-byte boundaries and
// strides are multiples of 16 bytes, so whole vectors are aligned; the last, partial one is fetched in pieces of
// four, two and one elements (nothing past the row's end is read).
template <bool kF32>
__device__ __forceinline__ Raw8<kF32> load8(const void* row, int c, int d) {
  Raw8<kF32> r;
  const int n = d - c;
  const char* at = static_cast<const char*>(row) + static_cast<size_t>(c) * (kF32 ? 4 : 2);
  if (n >= 8) {
    r.q[0] = *reinterpret_cast<const uint4*>(at);
    if (kF32) r.q[kF32 ? 1 : 0] = reinterpret_cast<const uint4*>(at)[1];
    return r;
  }
  r = zero8<kF32>();
  if (n <= 0) return r;
  if (kF32) {
    const uint32_t* e = reinterpret_cast<const uint32_t*>(at);
    uint4 tail = make_uint4(0u, 0u, 0u, 0u);  // the last n % 4
    const uint32_t* f = e + (n & 4);
    if (n & 2) {
      const uint2 u = *reinterpret_cast<const uint2*>(f);
      tail.x = u.x;
      tail.y = u.y;
      if (n & 1) tail.z = f[2];
    } else if (n & 1) {
      tail.x = f[0];
    }
    if (n & 4) {
      r.q[0] = *reinterpret_cast<const uint4*>(e);
      r.q[kF32 ? 1 : 0] = tail;
    } else {
      r.q[0] = tail;
    }
  } else {
    uint32_t lo = 0u, hi = 0u;  // the last n % 4
    const uint16_t* f = reinterpret_cast<const uint16_t*>(at) + (n & 4);
    if (n & 2) {
      lo = *reinterpret_cast<const uint32_t*>(f);
      if (n & 1) hi = f[2];
    } else if (n & 1) {
      lo = f[0];
    }
    if (n & 4) {
      const uint2 u = *reinterpret_cast<const uint2*>(at);
      r.q[0] = make_uint4(u.x, u.y, lo, hi);
    } else {
      r.q[0] = make_uint4(lo, hi, 0u, 0u);
    }
  }
  return r;
}
// The same for a prefetch, which must not touch what it loads: whole 16-byte pieces with an element of the row in
// them (n = d - c elements are left of it).  A piece that also reaches past the row's end lies in the row's own stride,
// but for the last row, whose partial piece is left out; trim8 brings a partial vector in order when it is used.
template <bool kF32, bool kRagged>
__device__ __forceinline__ Raw8<kF32> fetch8(const void* row, int c, int n, bool last) {
  Raw8<kF32> r = zero8<kF32>();
  const uint4* at = reinterpret_cast<const uint4*>(static_cast<const char*>(row) + static_cast<size_t>(c) * (kF32 ? 4 : 2));
  constexpr int kPer = kF32 ? 4 : 8;
  const int over = kRagged && last ? kPer - 1 : 0;
  if (n > over) r.q[0] = at[0];
  if (kF32) {
    if (n > (kRagged ? kPer + over : 0)) r.q[kF32 ? 1 : 0] = at[1];
  }
  return r;
}
// For 0 < d - c < 8.
template <bool kF32>
__device__ __forceinline__ void trim8(Raw8<kF32>& r, const void* row, int c, int d, bool last) {
  if (last) {
    r = load8<kF32>(row, c, d);
    return;
  }
  const int n = d - c;
  if (kF32) {
    uint4& a = r.q[0];
    uint4& b = r.q[kF32 ? 1 : 0];
    a.y = n > 1 ? a.y : 0u;
    a.z = n > 2 ? a.z : 0u;
    a.w = n > 3 ? a.w : 0u;
    b.x = n > 4 ? b.x : 0u;
    b.y = n > 5 ? b.y : 0u;
    b.z = n > 6 ? b.z : 0u;
    b.w = 0u;
  } else {
    auto keep = [&](uint32_t w, int i) { return n > i + 1 ? w : (n > i ? w & 0xffffu : 0u); };
    r.q[0] = make_uint4(keep(r.q[0].x, 0), keep(r.q[0].y, 2), keep(r.q[0].z, 4), keep(r.q[0].w, 6));
  }
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
// Stores them, those below d (kRagged: d may lie inside the vector).
template <bool kF32, bool kRagged = true>
__device__ __forceinline__ void store8(void* row, int c, int d, const V8& a) {
  const int n = kRagged ? d - c : (c < d ? 8 : 0);
  if (kF32) {
    float* p = static_cast<float*>(row) + c;
    if (n >= 8) {
      reinterpret_cast<float4*>(p)[0] = make_float4(a.v[0], a.v[1], a.v[2], a.v[3]);
      reinterpret_cast<float4*>(p)[1] = make_float4(a.v[4], a.v[5], a.v[6], a.v[7]);
    } else if (n > 0) {
      if (n & 4) *reinterpret_cast<float4*>(p) = make_float4(a.v[0], a.v[1], a.v[2], a.v[3]);
      float* f = p + (n & 4);
      if (n & 2) *reinterpret_cast<float2*>(f) = n & 4 ? make_float2(a.v[4], a.v[5]) : make_float2(a.v[0], a.v[1]);
      if (n & 1) p[n - 1] = n & 4 ? (n & 2 ? a.v[6] : a.v[4]) : (n & 2 ? a.v[2] : a.v[0]);
    }
  } else {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(row) + c;
    const uint32_t w[4] = {pack_bf16x2(a.v[0], a.v[1]), pack_bf16x2(a.v[2], a.v[3]), pack_bf16x2(a.v[4], a.v[5]),
                           pack_bf16x2(a.v[6], a.v[7])};
    if (n >= 8) {
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else if (n > 0) {
      if (n & 4) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
      const uint32_t lo = n & 4 ? w[2] : w[0], hi = n & 4 ? w[3] : w[1];  // the last n % 4
      if (n & 2) *reinterpret_cast<uint32_t*>(p + (n & 4)) = lo;
      if (n & 1) reinterpret_cast<uint16_t*>(p)[n - 1] = static_cast<uint16_t>(n & 2 ? hi : lo);
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
template <bool kF32, bool kRagged = true>
__device__ __forceinline__ void store8(void* row, int c, int d, const P8& a) {
  V8 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 q = unpair2(a.p[i]);
    v.v[2 * i] = q.x;
    v.v[2 * i + 1] = q.y;
  }
  store8<kF32, kRagged>(row, c, d, v);
}

// ---- a ring of rows in shared memory, filled by asynchronous copies; slot s of a stage holds 16 bytes of every
// thread, and every thread copies and reads only its own, so the ring needs no barrier ----
// 16 bytes, of which the first `bytes` are read and the others filled with zeros.
__device__ __forceinline__ void async_copy16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
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
// kWide: the block may have more than 16 warps.  kNarrow: sums over `span` neighbouring threads instead, without a barrier.
template <int N, bool kWide, bool kNarrow>
__device__ __forceinline__ void block_sum(float (&s)[N], SumBuf<N>& buf, int span) {
  if (kNarrow) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      if (o >= 8 && o >= span) continue;  // the same for the whole grid
#pragma unroll
      for (int k = 0; k < N; ++k) s[k] += __shfl_xor_sync(0xffffffffu, s[k], o);
    }
    return;
  }
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

// Forward.  kVec vectors of eight per thread; vector j of a thread starts at 8 * (its number in the row + j * blockDim).
// kGate: with kVec == 1 every token has a gate of its own (else none has); otherwise the call says.  kRagged: d need
// not be a multiple of 8.  Neither is carried along where it is not needed (d = 728, T = 65,536, bf16: 69 us; with the
// tests for a ragged row 87 us, with both decided at run time 94 us).  kNarrow: see norm_cfg (d = 64, T = 65,536:
// 8.2 us; a block of one warp per row took 40 us).
template <bool kF32, int kVec, int kThreads, bool kGate, bool kRagged, bool kNarrow>
__global__ void __launch_bounds__(kThreads, kVec == 1 ? 1024 / kThreads : 1) norm_fwd_kernel(const NormParams p) {
  __shared__ SumBuf<1> red[4];
  constexpr bool kHold = kVec == 1;  // gains held in registers, the next row's loads in flight
  constexpr bool kWide = kThreads > 512;
  // 1024 threads of 64 registers do not hold an fp32 row with its gate and the next ones: only x comes a row ahead,
  // gate and residual with the row (d = 8192, T = 10,000: 188 us; all of it ahead, with spills, 255 us)
  constexpr bool kLate = kHold && kWide && kF32 && kGate;
  constexpr size_t es = kF32 ? 4 : 2;
  const int nt = blockDim.x;
  const int span = kNarrow ? p.span : nt, sub = kNarrow ? static_cast<int>(threadIdx.x) / span : 0, rows = kNarrow ? nt / span : 1;
  const int col0 = 8 * (static_cast<int>(threadIdx.x) - sub * span);
  const float inv_d = 1.f / static_cast<float>(p.d);
  const bool token_gate = kGate && (kHold || (p.gate != nullptr && p.ldg != 0));
  P8 wp[kVec], wq[kVec];  // gain of the branch times a shared gate; gain of y
  grid_dependency_wait();
  grid_launch_dependents();
  auto gains = [&](int j) {
    const int c = col0 + 8 * j * nt;
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
  if (!kNarrow) {
    clear_sums(red, 4);
    __syncthreads();
  }
  struct Row {
    Raw8<false> x[kVec], g[kVec];
    Raw8<kF32> r[kVec];
  };
  auto x_row = [&](int t) { return p.x + static_cast<size_t>(t) * p.ldx; };
  auto r_row = [&](int t) { return static_cast<const char*>(p.residual) + static_cast<size_t>(t) * p.ldr * es; };
  auto g_row = [&](int t) { return p.gate + static_cast<size_t>(t) * p.ldg; };
  auto fetch = [&](int t) {
    Row o;
    const bool last = t == p.T - 1;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = col0 + 8 * j * nt, n = kNarrow && t >= p.T ? 0 : p.d - c;
      o.x[j] = p.x != nullptr ? fetch8<false, kRagged>(x_row(t), c, n, last) : zero8<false>();
      if (!kLate) o.r[j] = p.residual != nullptr ? fetch8<kF32, kRagged>(r_row(t), c, n, last) : zero8<kF32>();
      if (token_gate && !kLate) o.g[j] = fetch8<false, kRagged>(g_row(t), c, n, last);
    }
    return o;
  };
  const int step = static_cast<int>(gridDim.x) * rows;
  int par = 0;
  Row next;
  if (kHold && static_cast<int>(blockIdx.x) * rows < p.T) next = fetch(static_cast<int>(blockIdx.x) * rows + sub);
  for (int t0 = static_cast<int>(blockIdx.x) * rows; t0 < p.T; t0 += step, par ^= 1) {
    const int t = t0 + sub;
    const int lim = kNarrow && t >= p.T ? 0 : p.d;  // columns below it are stored
    Row cur = kHold ? next : fetch(t);
    if (kLate) {
      cur.g[0] = fetch8<false, kRagged>(g_row(t), col0, p.d - col0, t == p.T - 1);
      cur.r[0] = p.residual != nullptr ? fetch8<kF32, kRagged>(r_row(t), col0, p.d - col0, t == p.T - 1) : zero8<kF32>();
    }
    if (kHold && t0 + step < p.T) next = fetch(t + step);
    if (kRagged) {
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const int c = col0 + 8 * j * nt;
        if (c >= lim || c + 8 <= lim) continue;
        const bool last = t == p.T - 1;
        if (p.x != nullptr) trim8<false>(cur.x[j], x_row(t), c, p.d, last);
        if (p.residual != nullptr) trim8<kF32>(cur.r[j], r_row(t), c, p.d, last);
        if (token_gate) trim8<false>(cur.g[j], g_row(t), c, p.d, last);
      }
    }
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
      block_sum<1, kWide, kNarrow>(s, red[2 * par], span);
      scale *= rsqrtf(fmaf(s[0], inv_d, p.eps));
    }
    const unsigned long long scale2 = pair2(scale, scale), res2 = pair2(p.res_scale, p.res_scale);
    unsigned long long q = 0ull;
    P8 h[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = col0 + 8 * j * nt;
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
      if (p.h != nullptr)
        store8<kF32, kRagged>(static_cast<char*>(p.h) + static_cast<size_t>(t) * p.ldh * es, c, lim, h[j]);
    }
    if (p.y == nullptr) continue;
    float s[1] = {sum2(q)};
    block_sum<1, kWide, kNarrow>(s, red[2 * par + 1], span);
    const float rh = rsqrtf(fmaf(s[0], inv_d, p.eps));
    const unsigned long long rh2 = pair2(rh, rh);
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      P8 o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o.p[i] = mul2(mul2(h[j].p[i], rh2), wq[j].p[i]);
      store8<false, kRagged>(p.y + static_cast<size_t>(t) * p.ldy, col0 + 8 * j * nt, lim, o);
    }
  }
}

// Backward.  With G = b gate gain_post, v = dh G, and the sums over rows behind the gains and a shared gate are
// d_post = b gate S and d_gate = b gain_post S with the same S = sum_t dh x r_x (times the row's gate, if
// every token has its own), so a column needs two sums and two gains.  kVec == 1: they stay in registers, and the
// next rows' loads are in flight during the reductions: with a bf16 stream in a ring of kRing stages in shared memory
// (asynchronous copies, which take no registers), with an fp32 stream the next row in registers (d = 4096, T = 20,000:
// 252 us with it, 347 without; a ragged row is faster without, d = 300: 107 us against 120).  That
// takes up to 128 registers and leaves 512 threads per SM, which is enough once the loads are ahead: cut down to 80
// registers for 768 threads, the kernel spills (d = 1536, T = 53,328, bf16: 212 us against 167).
// kVec == 2: sums and gains in shared memory (dynamic, [2][d] each; d = 8192, T = 10,000: 254 us, with the gains read
// from memory and put together for each row 338 us; rows in a ring as well: no faster, so it is not the loads
// that they wait for).  kVec == 4: only the sums fit, gains are re-read.
// kForm > 0: every operand and result exists, and with kGate every token has its own gate (without it none has).  2: d
// is a multiple of 8 besides (no vector is partly outside the row); 3: of 256 (no thread is; d = 2048, T = 40,000: 160 us,
// as form 2 172 us, as form 1 170; an fp32 stream as form 1 296 us instead of 228).  kVec > 1: 2 or 0 (d = 8192, T =
// 10,000: 234 us as form 2, 254 as form 0; d = 12,288, T = 6664: 434 and 572 us).  A call with a missing part takes
// form 0, which tests for it and has nothing in flight ahead (a per-token gate at d = 1536, T = 53,328: 372 us in form 0, 202 us
// in its own; the norm in front of an LM head, where no gradient arrives at h from elsewhere, T = 8192, bf16: d = 1536
// 52 us, d = 4096 129 us, 37 and 40 % of the copy rate).
// kNarrow: see norm_cfg (d = 128, T = 65,536, bf16: 23 us; a block of one warp per row took 41 us).
template <bool kF32, int kVec, int kForm, bool kGate, int kThreads, bool kNarrow>
__global__ void __launch_bounds__(kThreads, 512 / kThreads) norm_bwd_kernel(const NormParams p) {
  __shared__ SumBuf<3> red3[2];
  __shared__ SumBuf<1> red1[2];
  extern __shared__ __align__(16) float dyn[];  // sums over rows, or the ring
  constexpr bool kHold = kVec == 1, kFull = kForm > 0, kRagged = kForm < 2;
  constexpr bool kRows = kHold && kFull && !kF32;  // rows arrive through the ring
  constexpr bool kKept = kVec == 2;       // gains kept in shared memory
  constexpr int kRing = norm_cfg::kRing;
  constexpr bool kNext = kHold && kFull && kF32 && !kRagged;  // the next row is in flight in registers
  constexpr size_t es = kF32 ? 4 : 2;
  const int nt = blockDim.x;
  const int span = kNarrow ? p.span : nt, sub = kNarrow ? static_cast<int>(threadIdx.x) / span : 0, rows = kNarrow ? nt / span : 1;
  const int col0 = 8 * (static_cast<int>(threadIdx.x) - sub * span);
  const float inv_d = 1.f / static_cast<float>(p.d);
  const bool shared_gate = !(kFull && kGate) && p.gate != nullptr && p.ldg == 0;
  const bool token_gate = kFull ? kGate : p.gate != nullptr && p.ldg != 0;
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
  ulonglong2* kept = sums + 4 * kVec * nt;  // kKept: the gains, in the same order
  auto gain = [&](int which, int j) {
    if (kHold) return held[which];
    if (!kKept) return read_gain(which, col0 + 8 * j * nt);
    P8 o;
    const ulonglong2* q = kept + 2 * (which * kVec + j) * nt + threadIdx.x;
    const ulonglong2 lo = q[0], hi = q[nt];
    o.p[0] = lo.x;
    o.p[1] = lo.y;
    o.p[2] = hi.x;
    o.p[3] = hi.y;
    return o;
  };
  if (!kNarrow) {
    clear_sums(red3, 2);
    clear_sums(red1, 2);
  }
  grid_dependency_wait();
  if (kHold) {
    held[0] = read_gain(0, col0);
    held[1] = read_gain(1, col0);
  } else {
    // every thread clears, adds to and reads back its own columns only: no barrier needed
    for (int i = 0; i < 4 * kVec; ++i) sums[i * nt + threadIdx.x] = make_ulonglong2(0ull, 0ull);
    if (kKept) {
#pragma unroll
      for (int w = 0; w < 2 * kVec; ++w) {
        const P8 v = read_gain(w / kVec, col0 + 8 * (w % kVec) * nt);
        for (int half = 0; half < 2; ++half)
          kept[(2 * w + half) * nt + threadIdx.x] = make_ulonglong2(v.p[2 * half], v.p[2 * half + 1]);
      }
    }
  }
  if (!kNarrow) __syncthreads();
  struct Row {
    Raw8<false> dy[kVec], x[kVec], g[kVec];
    Raw8<kF32> h[kVec], dh[kVec];
  };
  auto dy_row = [&](int t) { return p.dy + static_cast<size_t>(t) * p.lddy; };
  auto x_row = [&](int t) { return p.x + static_cast<size_t>(t) * p.ldx; };
  auto g_row = [&](int t) { return p.gate + static_cast<size_t>(t) * p.ldg; };
  auto h_row = [&](int t) { return static_cast<const char*>(p.h) + static_cast<size_t>(t) * p.ldh * es; };
  auto dh_row = [&](int t) { return static_cast<const char*>(p.dh) + static_cast<size_t>(t) * p.lddh * es; };
  const bool active = kForm == 3 || col0 < p.d;  // kHold: this thread has columns of the row
  auto fetch = [&](int t) {
    Row o;
    const bool last = t == p.T - 1;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = col0 + 8 * j * nt, n = kNarrow && t >= p.T ? 0 : (kForm == 3 ? 8 : p.d - c);
      o.dy[j] = have_y ? fetch8<false, kRagged>(dy_row(t), c, n, last) : zero8<false>();
      o.h[j] = have_y ? fetch8<kF32, kRagged>(h_row(t), c, n, last) : zero8<kF32>();
      o.dh[j] = have_dh ? fetch8<kF32, kRagged>(dh_row(t), c, n, last) : zero8<kF32>();
      o.x[j] = have_x ? fetch8<false, kRagged>(x_row(t), c, n, last) : zero8<false>();
      if (token_gate) o.g[j] = fetch8<false, kRagged>(g_row(t), c, n, last);
    }
    return o;
  };
  auto trim = [&](Row& o, int t) {
    const bool last = t == p.T - 1;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = col0 + 8 * j * nt;
      if (c >= p.d || c + 8 <= p.d || (kNarrow && t >= p.T)) continue;
      if (have_y) trim8<false>(o.dy[j], dy_row(t), c, p.d, last);
      if (have_y) trim8<kF32>(o.h[j], h_row(t), c, p.d, last);
      if (have_dh) trim8<kF32>(o.dh[j], dh_row(t), c, p.d, last);
      if (have_x) trim8<false>(o.x[j], x_row(t), c, p.d, last);
      if (token_gate) trim8<false>(o.g[j], g_row(t), c, p.d, last);
    }
  };
  // the ring: slots of a stage are dy, x, h, dh and a per-token gate
  constexpr int kSlots = kGate ? 5 : 4;
  const uint32_t slot = 16u * static_cast<uint32_t>(nt), ring0 = smem_u32(dyn) + 16u * threadIdx.x;
  const uint32_t bytes = kRagged ? static_cast<uint32_t>(min(16, 2 * (p.d - col0))) : 16u;
  auto issue = [&](int t, int stage) {
    if (t < p.T && active) {
      const uint32_t at = ring0 + static_cast<uint32_t>(stage) * kSlots * slot;
      async_copy16(at, dy_row(t) + col0, bytes);
      async_copy16(at + slot, x_row(t) + col0, bytes);
      async_copy16(at + 2 * slot, h_row(t) + 2 * col0, bytes);
      async_copy16(at + 3 * slot, dh_row(t) + 2 * col0, bytes);
      if (kGate) async_copy16(at + 4 * slot, g_row(t) + col0, bytes);
    }
    async_commit();
  };
  auto take = [&](int stage, bool on) {
    Row o;
    if (!on) {
      o.dy[0].q[0] = o.x[0].q[0] = o.h[0].q[0] = o.dh[0].q[0] = o.g[0].q[0] = make_uint4(0u, 0u, 0u, 0u);
      return o;
    }
    const uint32_t at = ring0 + static_cast<uint32_t>(stage) * kSlots * slot;
    o.dy[0].q[0] = ring_get(at);
    o.x[0].q[0] = ring_get(at + slot);
    o.h[0].q[0] = ring_get(at + 2 * slot);
    o.dh[0].q[0] = ring_get(at + 3 * slot);
    if (kGate) o.g[0].q[0] = ring_get(at + 4 * slot);
    return o;
  };
  const unsigned long long rs2 = pair2(p.res_scale, p.res_scale);
  const int step = static_cast<int>(gridDim.x) * rows;
  int par = 0, stage = 0;
#pragma unroll
  for (int i = 0; i < (kRows ? kRing : 0); ++i) issue(static_cast<int>(blockIdx.x) * rows + sub + i * step, i);
  Row next;
  if (kNext && static_cast<int>(blockIdx.x) * rows < p.T) next = fetch(static_cast<int>(blockIdx.x) * rows + sub);
  for (int t0 = static_cast<int>(blockIdx.x) * rows; t0 < p.T; t0 += step, par ^= 1) {
    const int t = t0 + sub;
    const bool on = active && (!kNarrow || t < p.T);
    const int lim = kNarrow && t >= p.T ? 0 : (kForm == 3 ? 1 << 30 : p.d);  // columns below it are stored
    Row cur;
    if (kRows) {
      async_wait<kRing - 1>();
      cur = take(stage, on);
    } else {
      cur = kNext ? next : fetch(t);
      if (kNext && t0 + step < p.T) next = fetch(t + step);
      if (kRagged) trim(cur, t);
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
      issue(t + kRing * step, stage);
      stage = stage + 1 == kRing ? 0 : stage + 1;
    }
    float s[3] = {sum2(s0), sum2(s1), sum2(s2)};  // sum h^2, sum g h, sum x^2
    block_sum<3, false, kNarrow>(s, red3[par], span);
    const float rh = have_y ? rsqrtf(fmaf(s[0], inv_d, p.eps)) : 0.f;
    const float rx = p.post ? rsqrtf(fmaf(s[2], inv_d, p.eps)) : 1.f;
    const float ch = -rh * rh * s[1] * inv_d;
    const unsigned long long rh2 = pair2(rh, rh), ch2 = pair2(ch, ch), rx2 = pair2(rx, rx);
    unsigned long long q = 0ull;  // sum v x
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = col0 + 8 * j * nt;
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
          if (!kNarrow || on) {  // a row beyond the last: its zeros times a reciprocal norm need not be zeros (eps = 0)
            acc[0].p[i] = fma2(mul2(dy.p[i], h.p[i]), rh2, acc[0].p[i]);
            acc[1].p[i] = fma2(d2, xn, acc[1].p[i]);
          }
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
      if (kFull || p.dres != nullptr)
        store8<kF32, kRagged>(static_cast<char*>(p.dres) + static_cast<size_t>(t) * p.lddres * es, c, lim, o);
      if (token_gate && (kFull || p.dgate != nullptr))
        store8<false, kRagged>(p.dgate + static_cast<size_t>(t) * p.lddgate, c, lim, dg);
    }
    if (!kFull && p.dx == nullptr) continue;
    if (p.post) {
      float sq[1] = {sum2(q)};
      block_sum<1, false, kNarrow>(sq, red1[par], span);
      const float cx = -rx * rx * sq[0] * inv_d;
      const unsigned long long cx2 = pair2(cx, cx);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const P8 x = pairs8<false>(cur.x[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) vv[j].p[i] = mul2(rx2, fma2(x.p[i], cx2, vv[j].p[i]));
      }
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j)
      store8<false, kRagged>(p.dx + static_cast<size_t>(t) * p.lddx, col0 + 8 * j * nt, lim, vv[j]);
  }
  grid_launch_dependents();
  if (p.want == 0) return;
  float* part = p.part + static_cast<size_t>(blockIdx.x) * 2 * p.part_d;
  if (kNarrow) {
    // the block's rows share columns: first the rows of a warp, then the warps, in a fixed order
    float f[2][8];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 v = unpair2(acc[a].p[i]);
        f[a][2 * i] = v.x;
        f[a][2 * i + 1] = v.y;
      }
#pragma unroll
    for (int o = 16; o >= 8; o >>= 1) {
      if (o < span) break;
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i >> 3][i & 7] += __shfl_xor_sync(0xffffffffu, f[i >> 3][i & 7], o);
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, cols = 8 * span, warps = nt >> 5;
    __syncthreads();  // the ring's memory is used again
    if (lane < span) {
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        float4* q = reinterpret_cast<float4*>(dyn + (2 * warp + a) * cols + 8 * lane);
        q[0] = make_float4(f[a][0], f[a][1], f[a][2], f[a][3]);
        q[1] = make_float4(f[a][4], f[a][5], f[a][6], f[a][7]);
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * cols; i += nt) {
      const int a = i >= cols ? 1 : 0, c = i - a * cols;
      if (c >= p.part_d) continue;
      float t = 0.f;
      for (int w = 0; w < warps; ++w) t += dyn[(2 * w + a) * cols + c];
      part[static_cast<size_t>(a) * p.part_d + c] = t;
    }
  } else if (kHold) {
    // rows of part_d floats: 16-byte stores; columns beyond d hold zeros
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int i = 0; i < 4; i += 2)
        if (col0 + 2 * i < p.part_d)
          *reinterpret_cast<ulonglong2*>(part + static_cast<size_t>(a) * p.part_d + col0 + 2 * i) = make_ulonglong2(acc[a].p[i], acc[a].p[i + 1]);
  } else {
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        for (int half = 0; half < 2; ++half) {
          const int c = col0 + 8 * j * nt + 4 * half;
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
