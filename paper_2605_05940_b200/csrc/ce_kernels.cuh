// Token cross-entropy of an LM head over a large vocabulary, and its gradient, without the [T, V]
// logits in memory:
//
//   z = H W^T / tau,  lse[t] = log sum_c exp z[t,c],  nll[t] = lse[t] - z[t, y_t]
//   dH = s (G W),  dW = s (G^T H),  G[t,c] = w_t (exp(z[t,c] - lse[t]) - [c = y_t]),  s = grad_scale / tau
//
// The tokens that count (mask set, label inside the vocabulary) are numbered and their hidden states
// gathered ("compact rows"); everything below works on those only.  Tensor-core tiles (pair_tile_sm100.cuh)
// form the logits twice: the forward tiles keep a running maximum and sum per row over a run of
// vocabulary tiles, and pick out the label's logit; the gradient tiles write G, in bf16, for one
// piece of the vocabulary at a time, and two contractions add the piece to dH and give its rows of dW.
// Logits are recomputed rather than kept: 8 d V operations per token for a method of 6 d V.
//
// Roundings: logits, maxima, sums and losses are fp32.  G is rounded to bf16 because the contractions'
// operands are; it holds w_t (p - [c = y]) without the scale s, which the contractions' epilogues
// multiply in fp32, so the label's entry is -1 but for a small p (exact in bf16 for w_t = 1) instead of
// one common rounding error of s in every token.
#pragma once

#include "pair_tile_sm100.cuh"
#include "rows_sm100.cuh"
#include "small_kernels.cuh"

namespace npd {

struct CePlanParams {
  int T, V, d;
  const uint8_t* mask;     // or NULL
  const int32_t* labels;
  const float* weight;     // token weights, or NULL
  const __nv_bfloat16* hidden;
  const __nv_bfloat16* head;
  long long ldh, ldw;
  float scale2;            // log2(e) / tau
  int vtiles, nsplit_max, clusters;
  int* plan;               // {blocks, pairs of blocks, forward runs, Tc}
  int* cidx;               // [T] compact row of a token, or -1
  int* cy;                 // [blocks*128] label of a compact row (-1 beyond Tc)
  float* cw;               // [blocks*128] weight of a compact row (0 beyond Tc)
  float* zy;               // [blocks*128] the label's scaled logit, summed in fp32 (see ce_merge_kernel)
  __nv_bfloat16* hc;       // [blocks*128, d] hidden states of the compact rows (0 beyond Tc with `pad`)
  float* dh_acc;           // [blocks*128, d], cleared here; or NULL
  int* status;
  int pad;
};

__device__ __forceinline__ bool ce_counts(const CePlanParams& p, int t) {
  if (p.mask != nullptr && p.mask[t] == 0) return false;
  const int y = p.labels[t];
  return y >= 0 && y < p.V;
}

// The number of forward runs (see choose_nsplit), the candidates tried by the lanes of one warp.
__device__ __forceinline__ int ce_choose_runs(int pairs, int vtiles, int clusters, int nsplit_max) {
  long long best = 1ll << 62;
  for (int ns = 1 + (threadIdx.x & 31); ns <= min(nsplit_max, vtiles); ns += 32) {
    const unsigned rounds = (static_cast<unsigned>(pairs) * ns + clusters - 1) / clusters, per = (vtiles + ns - 1) / ns;
    best = min(best, static_cast<long long>(rounds) * per * 128 + ns);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, o));
  return static_cast<int>(best % 128);  // ns < 128 here; a tie goes to fewer runs
}

// Numbers the tokens that count, in packed order, and gathers what the tiles read.  Every CTA handles a
// stretch of tokens; it counts the whole batch and the tokens before its stretch itself (5 bytes per token, from
// L2), which saves a second launch.  `pad`: the rows between Tc and the next multiple of 128 are cleared (the
// gradient's contractions multiply them by zeros).
__global__ void __launch_bounds__(1024) ce_plan_kernel(const CePlanParams p) {
  __shared__ int warp_n[2][32];
  __shared__ int list[1024];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  grid_dependency_wait();
  grid_launch_dependents();
  // stretches are whole multiples of 8 tokens
  const int grid = static_cast<int>(gridDim.x), block = static_cast<int>(blockIdx.x);
  const int per = ((p.T + grid - 1) / grid + 7) / 8 * 8;
  const int t0 = static_cast<int>(min(static_cast<long long>(p.T), static_cast<long long>(block) * per));
  const int t1 = min(p.T, t0 + per);
  int before = 0, all = 0;  // tokens that count: before t0, in the batch
  for (int t = threadIdx.x; t < p.T; t += blockDim.x) {
    const int one = ce_counts(p, t) ? 1 : 0;
    all += one;
    before += t < t0 ? one : 0;
  }
  before = warp_sum_int(before);
  all = warp_sum_int(all);
  if (lane == 0) {
    warp_n[0][warp] = before;
    warp_n[1][warp] = all;
  }
  __syncthreads();
  int base = warp_sum_int(warp_n[0][lane]);
  const int tc = warp_sum_int(warp_n[1][lane]);
  const int vecs = p.d / 8;
  for (int c0 = t0; c0 < t1; c0 += 1024) {
    const int t = c0 + static_cast<int>(threadIdx.x);
    const bool on = t < t1 && ce_counts(p, t);
    const unsigned votes = __ballot_sync(0xffffffffu, on);
    __syncthreads();  // the list and the warp counts of the round before have been read
    if (lane == 0) warp_n[0][warp] = __popc(votes);
    __syncthreads();
    const int mine = warp_n[0][lane], first = warp_sum_int(lane < warp ? mine : 0), n = warp_sum_int(mine);
    const int at = first + __popc(votes & ((1u << lane) - 1u));
    if (t < t1) p.cidx[t] = on ? base + at : -1;
    if (on) {
      list[at] = t;
      p.cy[base + at] = p.labels[t];
      p.cw[base + at] = p.weight != nullptr ? p.weight[t] : 1.f;
    }
    __syncthreads();
    // a warp per row: the hidden state, a clear row of the dH sums, and the label's logit in fp32
    for (int r = warp; r < n; r += 32) {
      const int tr = list[r];
      const uint4* src = reinterpret_cast<const uint4*>(p.hidden + static_cast<size_t>(tr) * p.ldh);
      uint4* dst = reinterpret_cast<uint4*>(p.hc + static_cast<size_t>(base + r) * p.d);
      for (int k = lane; k < vecs; k += 32) dst[k] = src[k];
      if (p.dh_acc != nullptr) {
        float4* acc = reinterpret_cast<float4*>(p.dh_acc + static_cast<size_t>(base + r) * p.d);
        for (int k = lane; k < 2 * vecs; k += 32) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      const float z = warp_dot_bf16(p.hidden + static_cast<size_t>(tr) * p.ldh, p.head + static_cast<size_t>(p.labels[tr]) * p.ldw, p.d, lane);
      if (lane == 0) p.zy[base + r] = z * p.scale2;
    }
    base += n;
  }
  const int nact = (tc + 127) / 128, pairs = (nact + 1) / 2;
  if (block == 0) {
    for (int i = tc + static_cast<int>(threadIdx.x); i < nact * 128; i += static_cast<int>(blockDim.x)) {
      p.cy[i] = -1;
      p.cw[i] = 0.f;
    }
    if (warp == 0) {
      const int runs = ce_choose_runs(pairs > 0 ? pairs : 1, p.vtiles, p.clusters, p.nsplit_max);
      if (lane == 0) {
        p.plan[0] = nact;
        p.plan[1] = pairs;
        p.plan[2] = runs;
        p.plan[3] = tc;
        *p.status = 0;
      }
    }
  }
  if (!p.pad) return;
  for (int r = tc + block * 32 + warp; r < nact * 128; r += grid * 32) {
    uint4* dst = reinterpret_cast<uint4*>(p.hc + static_cast<size_t>(r) * p.d);
    for (int k = lane; k < vecs; k += 32) dst[k] = make_uint4(0u, 0u, 0u, 0u);
    if (p.dh_acc != nullptr) {
      float4* acc = reinterpret_cast<float4*>(p.dh_acc + static_cast<size_t>(r) * p.d);
      for (int k = lane; k < 2 * vecs; k += 32) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
}

struct CeTileParams {
  int V, ksteps;
  const int* plan;
  const int* cy;       // [blocks*128]
  const float* cw;     // [blocks*128]
  int group_pairs;     // pairs of row blocks per group (see CeWalk)
  int vt_begin, vt_count;
  float scale2;        // log2(e) / tau
  long long rows;      // stride of the partials: compact rows the workspace has room for
  float2* partials;    // forward: [4 * runs][rows] {maximum, sum}, base 2, logits scaled by scale2
  float* zlabel;       // forward: [rows] the label's scaled logit
  const float* lse2;   // gradient: [rows] log2-sum-exp2 of the scaled logits
  __nv_bfloat16* gbuf; // gradient: scratch block [rows, ldg], 1024-byte aligned, ldg a multiple of 256
  long long ldg;
  int g_col0;          // gradient: vocabulary column of the scratch's column 0
  int* status;
};

// Units of (pair of row blocks, run of vocabulary tiles), dealt round robin.  They are ordered in
// groups of pairs whose hidden states fit a quarter of L2 (within a group the pair varies fastest, then
// the run), so the pairs that work at the same time share the W tiles in L2 and their H rows stay there.
// The forward cuts the vocabulary into plan[2] runs, the gradient into single tiles.
template <bool kRuns>
struct CeWalk {
  int pairs, nsplit, units, u, step, vt, vt1, row0, run, group, vt_begin, vt_count;
  bool fresh;
  __device__ __forceinline__ CeWalk(const CeTileParams& p, int pair, int num_pairs) {
    pairs = p.plan[1];
    nsplit = kRuns ? p.plan[2] : p.vt_count;
    units = pairs * nsplit;
    u = pair - num_pairs;
    step = num_pairs;
    vt = vt1 = row0 = run = 0;
    group = max(1, min(p.group_pairs, pairs));
    vt_begin = p.vt_begin;
    vt_count = p.vt_count;
    fresh = false;
  }
  __device__ __forceinline__ bool next(PairTile& t) {
    if (vt >= vt1) {
      u += step;
      if (u >= units) return false;
      const int per_group = group * nsplit;
      const int gi = u / per_group, local = u - gi * per_group;
      const int gsize = min(group, pairs - gi * group);
      run = local / gsize;
      row0 = 256 * (gi * group + local % gsize);
      vt = vt_begin + static_cast<int>(static_cast<long long>(vt_count) * run / nsplit);
      vt1 = vt_begin + static_cast<int>(static_cast<long long>(vt_count) * (run + 1) / nsplit);
      fresh = true;
    }
    t.row0 = row0;
    t.tile = vt++;
    t.run = run;
    t.first = fresh;
    t.last = vt >= vt1;
    fresh = false;
    return true;
  }
};

// Forward: running maximum and sum of the scaled logits of this thread's row over a run of tiles.
struct CeForwardEpi {
  using Params = CeTileParams;
  using Walk = CeWalk<true>;
  static constexpr int kBN = 256;
  static __device__ __forceinline__ int rows(const Params& p) { return 128 * p.plan[0]; }
  const Params& p;
  int pair_row, quarter, row, y, tc;
  float m, s;
  __device__ __forceinline__ CeForwardEpi(const Params& p_, int pair_row_, int quarter_)
      : p(p_), pair_row(pair_row_), quarter(quarter_), row(0), y(-1), tc(p_.plan[3]), m(-INFINITY), s(0.f) {}
  __device__ __forceinline__ void begin(const PairTile& t) {
    if (!t.first) return;
    row = t.row0 + pair_row;
    y = row < tc ? p.cy[row] : -1;
    m = -INFINITY;
    s = 0.f;
  }
  __device__ __forceinline__ void chunk(const uint32_t (&acc)[32], int col0) {
    const int nvalid = p.V - col0;
    if (nvalid <= 0) return;
    float z[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) z[i] = __uint_as_float(acc[i]) * p.scale2;
    if (nvalid < 32) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i >= nvalid) z[i] = -INFINITY;
    }
    const int yi = y - col0;
    if (static_cast<unsigned>(yi) < 32u) {  // the label is one of these columns (once per row)
      float zy = 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) zy = i == yi ? z[i] : zy;
      p.zlabel[row] = zy;
    }
    float c[4] = {z[0], z[1], z[2], z[3]};
#pragma unroll
    for (int i = 4; i < 32; ++i) c[i & 3] = fmaxf(c[i & 3], z[i]);
    const float top = fmaxf(fmaxf(c[0], c[1]), fmaxf(c[2], c[3]));
    if (top > m) {
      s *= ex2f(m - top);
      m = top;
    }
    // a row of -inf so far (or of NaN): subtracting it from itself would make NaN out of -inf
    const float base = m == -INFINITY ? 0.f : m;
    float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 32; ++i) a[i & 3] += ex2f(z[i] - base);
    s += (a[0] + a[1]) + (a[2] + a[3]);
  }
  __device__ __forceinline__ void end(const PairTile& t) {
    if (t.last && row < tc) p.partials[static_cast<size_t>(4 * t.run + quarter) * p.rows + row] = make_float2(m, s);
  }
};

// The forward for few tokens (at most 8): the tiles above would spend 256 rows of tensor memory and operand stages on
// them, and take longer than reading the weights (T = 1: 157 us at d = 1536 and 300 us at d = 4096, V = 151,936).  A
// block takes 16 vocabulary rows at a time (rows_sm100.cuh), one group after the other across the whole grid;
// every (token, row of 16) has a thread that keeps a running maximum and sum of the logits it sees.  They are merged
// over the block at its end, and over the blocks by ce_merge_kernel.  The instruction holds 8 tokens; from 9 on the tiles
// take over, which are slower at first (the whole forward at V = 151,936: T = 8 85 us at d = 1536 and 203 at d = 4096, T = 9 112 and
// 284, T = 32 118 and 256, T = 64 104 at d = 1536).
struct CeRowsParams {
  int V, d;
  const int* plan;
  const int* cy;
  const __nv_bfloat16* hc;      // [128, d], anything beyond Tc: tokens do not mix
  const __nv_bfloat16* weight;
  long long ldw, rows;
  float scale2;
  float2* partials;             // [gridDim][rows]
  float* zlabel;
};

__device__ __forceinline__ float2 merge_max_sum(float2 a, float2 b) {
  const float top = fmaxf(a.x, b.x), base = top == -INFINITY ? 0.f : top;
  return make_float2(top, a.y * ex2f(a.x - base) + b.y * ex2f(b.x - base));
}

template <int kBatch>
__global__ void __launch_bounds__(ce_rows_cfg::kThreads, kBatch == 3 ? 3 : 2) ce_rows_kernel(const CeRowsParams p) {
  using namespace ce_rows_cfg;
  __shared__ float part[2][kWarps][kTokens][17];  // [..][row of 16], padded against bank conflicts
  extern __shared__ __align__(16) unsigned char xs[];  // [step][lane]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
  grid_dependency_wait();
  grid_launch_dependents();
  const int tc = p.plan[3];
  if (tc == 0) return;
  const int steps = p.d / 32, s0 = steps * warp / kWarps, s1 = steps * (warp + 1) / kWarps;
  for (int s = s0; s < s1; ++s)
    *reinterpret_cast<uint4*>(xs + static_cast<size_t>(s) * 512 + 16 * lane) =
        *reinterpret_cast<const uint4*>(p.hc + static_cast<size_t>(g) * p.d + s * 32 + 8 * q);
  // the first 128 threads: token threadIdx / 16, row threadIdx % 16
  const int token = threadIdx.x >> 4, row = threadIdx.x & 15;
  const int y = token < kTokens ? p.cy[token] : -1;  // -1 beyond Tc
  float2 ms = make_float2(-INFINITY, 0.f);
  int buf = 0;
  rows_loop<kBatch>(p.weight, p.ldw, p.V, p.d, smem_u32(xs) + 512u * s0 + 16u * lane, 16 * blockIdx.x, 16 * gridDim.x, s0, s1,
                    [&](int r, const float (&acc)[4]) {
                      float(*o)[17] = part[buf][warp];
                      o[2 * q][g] = acc[0];
                      o[2 * q + 1][g] = acc[1];
                      o[2 * q][g + 8] = acc[2];
                      o[2 * q + 1][g + 8] = acc[3];
                      __syncthreads();  // two buffers: a warp that is ahead writes the other one
                      if (token < kTokens && r + row < p.V) {
                        float z = 0.f;
#pragma unroll
                        for (int w = 0; w < kWarps; ++w) z += part[buf][w][token][row];
                        z *= p.scale2;
                        if (r + row == y) p.zlabel[token] = z;
                        ms = merge_max_sum(ms, make_float2(z, 1.f));
                      }
                      buf ^= 1;
                    });
  // the sixteen rows of a token sit in half a warp
#pragma unroll
  for (int o = 1; o < 16; o <<= 1)
    ms = merge_max_sum(ms, make_float2(__shfl_xor_sync(0xffffffffu, ms.x, o), __shfl_xor_sync(0xffffffffu, ms.y, o)));
  if (row == 0 && token < kTokens && token < tc) p.partials[static_cast<size_t>(blockIdx.x) * p.rows + token] = ms;
}

// Gradient: G = w (p - [c = y]) in bf16 into the scratch block of this piece of the vocabulary.
struct CeGradientEpi {
  using Params = CeTileParams;
  using Walk = CeWalk<false>;
  static constexpr int kBN = 256;
  static __device__ __forceinline__ int rows(const Params& p) { return 128 * p.plan[0]; }
  const Params& p;
  int pair_row, tc, blocks128, y, row0;
  bool on;
  float w, lse2;
  __device__ __forceinline__ CeGradientEpi(const Params& p_, int pair_row_, int)
      : p(p_), pair_row(pair_row_), tc(p_.plan[3]), blocks128(128 * p_.plan[0]), y(-1), row0(-1), on(false), w(0.f), lse2(1e30f) {}
  __device__ __forceinline__ void begin(const PairTile& t) {
    if (t.row0 == row0) return;
    row0 = t.row0;
    const int row = row0 + pair_row;
    on = row < tc;
    y = on ? p.cy[row] : -1;
    w = on ? p.cw[row] : 0.f;
    lse2 = on ? p.lse2[row] : 0.f;
  }
  __device__ __forceinline__ void chunk(const uint32_t (&acc)[32], int col0) {
    if (row0 + pair_row >= blocks128) return;  // a block of rows that does not exist: nothing to store
    float g[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) g[i] = w * ex2f(fmaf(__uint_as_float(acc[i]), p.scale2, -lse2));
    const int yi = y - col0;
    if (static_cast<unsigned>(yi) < 32u) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i == yi) g[i] = w * (ex2f(fmaf(__uint_as_float(acc[i]), p.scale2, -lse2)) - 1.f);
    }
    const int nvalid = p.V - col0;
    // columns beyond V, and rows beyond the last token (whatever their logits), multiply real numbers: zeros
    if (nvalid < 32 || !on) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i >= nvalid || !on) g[i] = 0.f;
    }
    store_row32<false>(p.gbuf + static_cast<size_t>(row0 + pair_row) * p.ldg + (col0 - p.g_col0), g, 32, true);
  }
  __device__ __forceinline__ void end(const PairTile&) {}
};

struct CeMergeParams {
  int T;
  int slots;    // ce_merge_rows_kernel: partials per token (ce_merge_kernel: four per run of the tiles)
  const int* plan;
  const int* cidx;
  const float2* partials;
  long long rows;
  const float* zlabel;  // the label's scaled logit as the tiles have it
  const float* zy;      // and as the fp32 dot product has it
  float* nll;
  float* lse;   // or NULL
  float* lse2;  // [rows] for the gradient tiles
};

// Four partials into a running maximum and sum; the loads come first.
__device__ __forceinline__ float2 merge_four(float2 v, const float2 (&q)[4]) {
  const float top = fmaxf(fmaxf(fmaxf(q[0].x, q[1].x), fmaxf(q[2].x, q[3].x)), v.x), base = top == -INFINITY ? 0.f : top;
  float s = v.y * ex2f(v.x - base);
#pragma unroll
  for (int i = 0; i < 4; ++i) s = fmaf(q[i].y, ex2f(q[i].x - base), s);
  return make_float2(top, s);
}

// What a token's merged maximum and sum give.
// The tensor core cuts its partial sums instead of rounding them, so a logit is off by about 1e-6 of its
// size in one direction.  In the sum over a vocabulary that averages out; the label's logit stands alone.  It
// is therefore taken again as an fp32 dot product, and the difference e (that of the label's logit to
// the tiles' value) enters to first order: lse + p e, nll - (1 - p) e, p the label's probability.  e is
// around 1e-5, so the second order is below fp32.  (Subtracting an exact logit from an inexact lse
// instead would spoil the losses near 0, where the two are nearly equal.)
__device__ __forceinline__ void ce_write_token(const CeMergeParams& p, int t, int c, float2 v) {
  float nll = 0.f, lse = 0.f;
  if (c >= 0) {
    const float base = v.x == -INFINITY ? 0.f : v.x;
    const float l2 = base + log2f(v.y), zl = p.zlabel[c];
    const float e = p.zy[c] - zl, prob = ex2f(zl - l2);
    p.lse2[c] = l2;
    lse = kLn2 * fmaf(prob, e, l2);
    nll = kLn2 * fmaf(prob - 1.f, e, l2 - zl);
    nll = nll < 0.f ? 0.f : nll;  // rounding may dip below 0; NaN stays NaN
  }
  p.nll[t] = nll;
  if (p.lse != nullptr) p.lse[t] = lse;
}

// Merges the runs' maxima and sums into a token's log-sum-exp.  A block takes 32 tokens (one per lane,
// so that neighbouring compact rows are read together) and spreads the runs over its 8 warps.
__global__ void __launch_bounds__(256) ce_merge_kernel(const CeMergeParams p) {
  __shared__ float2 part[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = blockIdx.x * 32 + lane;
  grid_dependency_wait();
  grid_launch_dependents();
  const int c = t < p.T ? p.cidx[t] : -1;
  const int slots = 4 * p.plan[2];
  float2 v = make_float2(-INFINITY, 0.f);
  if (c >= 0) {
    for (int i = 4 * warp; i < slots; i += 32) {  // the four quarters of a run
      float2 q[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) q[u] = p.partials[static_cast<size_t>(i + u) * p.rows + c];
      v = merge_four(v, q);
    }
  }
  part[warp][lane] = v;
  __syncthreads();
  if (warp != 0 || t >= p.T) return;
#pragma unroll
  for (int w = 1; w < 8; ++w) v = merge_max_sum(v, part[w][lane]);
  ce_write_token(p, t, c, v);
}

// The same for the blocks of ce_rows_kernel: a block per token, the partials over its threads.
__global__ void __launch_bounds__(256) ce_merge_rows_kernel(const CeMergeParams p) {
  __shared__ float2 part[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = blockIdx.x;
  grid_dependency_wait();
  grid_launch_dependents();
  const int c = p.cidx[t];
  float2 v = make_float2(-INFINITY, 0.f);
  if (c >= 0)
    for (int i = threadIdx.x; i < p.slots; i += 256) v = merge_max_sum(v, p.partials[static_cast<size_t>(i) * p.rows + c]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    v = merge_max_sum(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
  if (lane == 0) part[warp] = v;
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int w = 1; w < 8; ++w) v = merge_max_sum(v, part[w]);
  ce_write_token(p, t, c, v);
}

// fp32 dH sums over the compact rows, times `scale` -> bf16 rows of the tokens; tokens that do not count
// get zeros.  8 elements per thread.
__global__ void __launch_bounds__(256) ce_scatter_kernel(const float* __restrict__ src, const int* __restrict__ cidx,
                                                        int T, int d, float scale, __nv_bfloat16* dst, long long ld) {
  grid_dependency_wait();
  grid_launch_dependents();
  const long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x;
  const int per_row = d / 8;
  if (i >= static_cast<long long>(T) * per_row) return;
  const int t = static_cast<int>(i / per_row), k = static_cast<int>(i % per_row) * 8;
  const int c = cidx[t];
  uint4 o = make_uint4(0u, 0u, 0u, 0u);
  if (c >= 0) {
    const float4 a = *reinterpret_cast<const float4*>(src + static_cast<size_t>(c) * d + k);
    const float4 b = *reinterpret_cast<const float4*>(src + static_cast<size_t>(c) * d + k + 4);
    o.x = pack_bf16x2(scale * a.x, scale * a.y);
    o.y = pack_bf16x2(scale * a.z, scale * a.w);
    o.z = pack_bf16x2(scale * b.x, scale * b.y);
    o.w = pack_bf16x2(scale * b.z, scale * b.w);
  }
  *reinterpret_cast<uint4*>(dst + static_cast<size_t>(t) * ld + k) = o;
}

}  // namespace npd
