// Products of a large weight matrix with up to 8 tokens, bound by reading the weights once, for a grid that stays
// resident and goes through many groups of rows.
//
// A block of 8 warps takes 16 rows of W at a time; its warps share out K, so that the block reads 16 whole
// rows, consecutive in memory (warps that read whole rows of their own scatter the block's reads over 128 rows, 64
// bytes at a time, and reached two thirds of the bandwidth).  mma.sync m16n8k16 with the 16 rows of W as one
// operand and the 8 tokens as the other: the tensor throughput does not matter at a handful of operations per byte,
// and this form takes its operands from registers, which every thread loads for itself; tcgen05 would want them
// staged in shared memory.  The order of the contraction is free: a thread's 16-byte vector of a row serves as
// the k indices that the instruction gives this thread in two successive MMAs, for W and x alike.
// The next batch of weights is loaded before the current one is used, across the boundary between groups of rows
// too; the tokens' vectors sit in shared memory, where every thread reads back what it wrote.
#pragma once

#include "linear_kernels.cuh"

namespace npd {

namespace ce_rows_cfg {
constexpr int kTokens = 8;
constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kMaxTokenBytes = 64 * 1024;  // shared memory for the tokens of a block (two blocks per SM)
}  // namespace ce_rows_cfg

template <int kBatch>
struct RowsBatch {
  uint4 a[kBatch], b[kBatch];  // rows lane/4 and lane/4 + 8
};
// Steps s.. (below s1) of the group of rows r.. (rows at or beyond N: the last row's values in their place).
template <int kBatch>
__device__ __forceinline__ void rows_load(RowsBatch<kBatch>& o, const __nv_bfloat16* w, long long ldw, int N, int K, int r, int s, int s1) {
  const int g = (threadIdx.x & 31) >> 2, q = threadIdx.x & 3;
  const __nv_bfloat16* w0 = w + static_cast<size_t>(min(r + g, N - 1)) * ldw;
  const __nv_bfloat16* w1 = w + static_cast<size_t>(min(r + g + 8, N - 1)) * ldw;
  if (s + kBatch <= s1 && (s + kBatch) * 32 <= K) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      o.a[u] = __ldg(reinterpret_cast<const uint4*>(w0 + (s + u) * 32 + 8 * q));
      o.b[u] = __ldg(reinterpret_cast<const uint4*>(w1 + (s + u) * 32 + 8 * q));
    }
  } else {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int k = s + u < s1 ? (s + u) * 32 + 8 * q : K;  // beyond: zeros
      o.a[u] = load8<false>(w0, k, K).q[0];
      o.b[u] = load8<false>(w1, k, K).q[0];
    }
  }
}

// Groups of 16 rows from r on, `stride` rows apart, below N; this warp's steps s0 .. s1-1.  xs: this thread's token
// vectors in shared memory, one per step, 512 bytes apart (a warp's vectors of a step lie together).
// done(r, acc) gets this warp's part of the group's products: thread (g, q) = (lane/4, lane%4) holds rows g and g + 8
// (acc[0..1], acc[2..3]) of tokens 2q and 2q + 1.
template <int kBatch, class Done>
__device__ __forceinline__ void rows_loop(const __nv_bfloat16* w, long long ldw, int N, int K, uint32_t xs, int r, int stride, int s0,
                                          int s1, Done done) {
  RowsBatch<kBatch> cur, next;
  if (r < N) rows_load<kBatch>(cur, w, ldw, N, K, r, s0, s1);
  for (; r < N; r += stride) {
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = s0; s < s1; s += kBatch) {
      const bool wrap = s + kBatch >= s1;
      const int nr = wrap ? r + stride : r, ns = wrap ? s0 : s + kBatch;
      if (nr < N) rows_load<kBatch>(next, w, ldw, N, K, nr, ns, s1);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        // beyond s1 the weights are zeros, and so are the tokens' products unless they are not finite: no product there
        if (s + u < s1) {
          const uint4 x = ring_get(xs + static_cast<uint32_t>(s + u - s0) * 512u);
          mma_16816(acc, cur.a[u].x, cur.b[u].x, cur.a[u].y, cur.b[u].y, x.x, x.y);
          mma_16816(acc, cur.a[u].z, cur.b[u].z, cur.a[u].w, cur.b[u].w, x.z, x.w);
        }
      }
      cur = next;
    }
    done(r, acc);
  }
}

}  // namespace npd
