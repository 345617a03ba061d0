// Host side of npd_ce_fwd_bwd.  Included by npd_api.cu, whose helpers it uses.
#pragma once

#include "ce_kernels.cuh"

namespace {

struct CePlan {
  int row_blocks, vtiles, clusters, nsplit_max, chunk_cols, nchunks;
  bool grads;
  size_t off_status, off_plan, off_cidx, off_cy, off_cw, off_hc, off_partials, off_zlabel, off_zy, off_lse2, off_g, off_dh, total;
};

CePlan ce_plan(const npd_ce_args* a, int sms) {
  CePlan pl{};
  pl.row_blocks = (a->T + 127) / 128;
  pl.vtiles = (a->V + 255) / 256;
  pl.clusters = std::max(sms / 2, 1);
  // As many runs as CTA pairs: a batch of one pair of row blocks (a few tokens to score) then still
  // has every SM reading its own part of the weights.  The partials cost 32 bytes per token and run.
  pl.nsplit_max = std::min({pl.vtiles, pl.clusters, 127});
  pl.grads = a->d_hidden != nullptr || a->d_weight != nullptr;
  // Pieces of the vocabulary in the backward: by default the widest whose bf16 gradient block stays
  // within 256 MiB or a sixteenth of what bf16 logits would take, whichever is more, all of (almost) equal width.
  const long long budget = std::max<long long>(256ll << 20, static_cast<long long>(a->T) * a->V / 8);
  int max_tiles = a->grad_chunk_cols > 0
                      ? static_cast<int>((static_cast<long long>(a->grad_chunk_cols) + 255) / 256)
                      : static_cast<int>(std::max<long long>(8, budget / (512ll * a->T)));
  max_tiles = std::max(1, std::min(max_tiles, pl.vtiles));
  pl.nchunks = (pl.vtiles + max_tiles - 1) / max_tiles;
  const int chunk_tiles = (pl.vtiles + pl.nchunks - 1) / pl.nchunks;
  pl.chunk_cols = chunk_tiles * 256;
  pl.nchunks = (pl.vtiles + chunk_tiles - 1) / chunk_tiles;
  const size_t crows = static_cast<size_t>(pl.row_blocks) * 128;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes, 1024);
    return at;
  };
  pl.off_status = take(1024);
  pl.off_plan = take(1024);
  pl.off_cidx = take(sizeof(int) * static_cast<size_t>(a->T));
  pl.off_cy = take(sizeof(int) * crows);
  pl.off_cw = take(sizeof(float) * crows);
  pl.off_hc = take(2 * crows * a->d);
  pl.off_partials = take(sizeof(float2) * std::max(4 * pl.nsplit_max, a->T <= ce_rows_cfg::kTokens ? 3 * sms : 0) * crows);
  pl.off_zlabel = take(sizeof(float) * crows);
  pl.off_zy = take(sizeof(float) * crows);
  pl.off_lse2 = take(sizeof(float) * crows);
  pl.off_g = pl.off_dh = off;
  if (pl.grads) {
    pl.off_g = take(2 * crows * pl.chunk_cols);
    if (a->d_hidden != nullptr) pl.off_dh = take(sizeof(float) * crows * a->d);
  }
  pl.total = off;
  return pl;
}

int check_ce(const npd_ce_args* a, bool need_pointers) {
  if (a == nullptr || a->size != sizeof(npd_ce_args)) return NPD_EINVAL;
  if (a->T < 1 || a->d < 1 || a->V < 1) return NPD_EINVAL;
  if (!(a->temperature > 0.f) || !std::isfinite(a->temperature) || !std::isfinite(a->grad_scale)) return NPD_EINVAL;
  if (a->d_weight_dtype != NPD_DTYPE_BF16 && a->d_weight_dtype != NPD_DTYPE_F32) return NPD_EINVAL;
  if ((a->flags & ~(NPD_CE_ACCUMULATE_DW | NPD_CE_SERIALIZE_LAUNCHES)) || a->grad_chunk_cols < 0) return NPD_EINVAL;
  if ((a->flags & NPD_CE_ACCUMULATE_DW) && a->d_weight_dtype != NPD_DTYPE_F32) return NPD_EINVAL;
  // Row numbers, columns, numbers of tiles and the bytes of eight tokens (ce_rows_kernel) are 32-bit.  A product of
  // 2^46 is at most 2^30 + (2^30 + 2^30) / 256 + 1 tiles of 256 x 256.
  if (a->T > (1 << 30) || a->V > (1 << 30) || a->d > (1 << 26)) return NPD_ESHAPE;
  const long long nt = a->T, nv = a->V, nd = a->d;
  if (std::max({nt * nv, nt * nd, nv * nd}) > 1ll << 46) return NPD_ESHAPE;
  if (a->d % 64 != 0) return NPD_ESHAPE;
  if (!need_pointers) return NPD_OK;
  if (a->hidden == nullptr || a->weight == nullptr || a->labels == nullptr || a->nll == nullptr) return NPD_EINVAL;
  const bool wf32 = a->d_weight_dtype == NPD_DTYPE_F32;
  struct M { const void* p; int64_t ld; int mult; };
  const M mats[] = {{a->hidden, a->ldh, 8}, {a->weight, a->ldw, 8}, {a->d_hidden, a->ld_dh, 8},
                    {a->d_weight, a->ld_dw, wf32 ? 4 : 8}};
  for (const M& m : mats) {
    if (m.p == nullptr) continue;
    if (m.ld < a->d) return NPD_ESHAPE;
    if (m.ld % m.mult || !aligned16(m.p)) return NPD_EALIGN;
  }
  for (const void* q : {static_cast<const void*>(a->labels), static_cast<const void*>(a->token_weight),
                        static_cast<const void*>(a->nll), static_cast<const void*>(a->lse)})
    if (reinterpret_cast<uintptr_t>(q) & 3) return NPD_EALIGN;
  // results apart from the operands and from each other (the pieces of the vocabulary re-read them)
  const long long T = a->T, V = a->V, d = a->d, we = wf32 ? 4 : 2;
  const Extent ins[] = {{a->hidden, T, 2 * d, 2 * a->ldh}, {a->weight, V, 2 * d, 2 * a->ldw}, {a->labels, 1, 4 * T, 4 * T},
                        {a->loss_mask, 1, T, T}, {a->token_weight, 1, 4 * T, 4 * T}};
  const Extent outs[] = {{a->nll, 1, 4 * T, 4 * T}, {a->lse, 1, 4 * T, 4 * T}, {a->d_hidden, T, 2 * d, 2 * a->ld_dh},
                         {a->d_weight, V, we * d, we * a->ld_dw}};
  for (int o = 0; o < 4; ++o) {
    for (const Extent& in : ins)
      if (extents_touch(outs[o], in)) return NPD_EINVAL;
    for (int q = o + 1; q < 4; ++q)
      if (extents_touch(outs[o], outs[q])) return NPD_EINVAL;
  }
  return NPD_OK;
}

// Launch of a pair-tile kernel: always one CTA pair per two SMs (at most `tiles` pairs when the host knows).
template <class Epi>
int launch_pair_tile(const CUtensorMap& ma, const CUtensorMap& mb, const typename Epi::Params& p, int pairs, cudaStream_t st,
                     bool pdl) {
  using L = PairCfg<Epi::kBN>;
  auto k = pair_tile_kernel<Epi>;
  if (set_smem(k, L::SMEM_BYTES) != NPD_OK) return NPD_ECUDA;
  const cudaError_t e = launch_ex(k, 2 * pairs, L::THREADS, L::SMEM_BYTES, st, pdl, ma, mb, p);
  ++g_launches;
  return e == cudaSuccess ? NPD_OK : NPD_ECUDA;
}

}  // namespace

extern "C" {

int npd_ce_workspace_bytes(const npd_ce_args* args, size_t* out_bytes) {
  if (out_bytes == nullptr) return NPD_EINVAL;
  int rc = check_ce(args, false);
  if (rc != NPD_OK) return rc;
  DeviceInfo di;
  if ((rc = device_info(&di)) != NPD_OK) return rc;
  *out_bytes = ce_plan(args, di.sms).total;
  return NPD_OK;
}

int npd_ce_fwd_bwd(const npd_ce_args* a, void* cuda_stream) {
  g_launches = 0;
  int rc = check_ce(a, true);
  if (rc != NPD_OK) return rc;
  DeviceInfo di;
  if ((rc = device_info(&di)) != NPD_OK) return rc;
  if (di.cc_major != 10) return NPD_EARCH;
  const CePlan pl = ce_plan(a, di.sms);
  if (a->workspace == nullptr || (reinterpret_cast<uintptr_t>(a->workspace) & 1023u) || a->workspace_bytes < pl.total)
    return NPD_EWORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  uint8_t* ws = static_cast<uint8_t*>(a->workspace);
  const bool pdl = (a->flags & NPD_CE_SERIALIZE_LAUNCHES) == 0;
  const uint64_t crows = static_cast<uint64_t>(pl.row_blocks) * 128;
  int* status = reinterpret_cast<int*>(ws + pl.off_status);
  __nv_bfloat16* hc = reinterpret_cast<__nv_bfloat16*>(ws + pl.off_hc);
  float* dh_acc = a->d_hidden != nullptr ? reinterpret_cast<float*>(ws + pl.off_dh) : nullptr;
  CUtensorMap mh, mw;
  // the compact rows end at T at the latest: rows of a tile beyond it are filled with zeros without a fetch
  if (!make_map(&mh, hc, a->d, a->T, a->d, 64, 128) || !make_map(&mw, a->weight, a->d, a->V, a->ldw, 64, 128))
    return NPD_ECUDA;

  CePlanParams pp{};
  pp.T = a->T;
  pp.V = a->V;
  pp.d = a->d;
  pp.mask = a->loss_mask;
  pp.labels = a->labels;
  pp.weight = a->token_weight;
  pp.hidden = static_cast<const __nv_bfloat16*>(a->hidden);
  pp.ldh = a->ldh;
  pp.head = static_cast<const __nv_bfloat16*>(a->weight);
  pp.ldw = a->ldw;
  pp.scale2 = 1.4426950408889634f / a->temperature;
  pp.vtiles = pl.vtiles;
  pp.nsplit_max = pl.nsplit_max;
  pp.clusters = pl.clusters;
  pp.plan = reinterpret_cast<int*>(ws + pl.off_plan);
  pp.cidx = reinterpret_cast<int*>(ws + pl.off_cidx);
  pp.cy = reinterpret_cast<int*>(ws + pl.off_cy);
  pp.cw = reinterpret_cast<float*>(ws + pl.off_cw);
  pp.zy = reinterpret_cast<float*>(ws + pl.off_zy);
  pp.hc = hc;
  pp.dh_acc = dh_acc;
  pp.status = status;
  pp.pad = pl.grads ? 1 : 0;
  // eight tokens per block or more; with rows to be cleared at least as many blocks as make that quick
  const int plan_blocks = std::min(di.sms, std::max((a->T + 7) / 8, pl.grads ? 4 : 1));
  if (launch_ex(ce_plan_kernel, plan_blocks, 1024, 0, st, false, pp) != cudaSuccess) return NPD_ECUDA;
  ++g_launches;

  CeTileParams tp{};
  tp.V = a->V;
  tp.ksteps = a->d / 64;
  tp.plan = pp.plan;
  tp.cy = pp.cy;
  tp.cw = pp.cw;
  tp.group_pairs = static_cast<int>(std::max<long long>(4, (32ll << 20) / (512ll * a->d)));
  tp.vt_begin = 0;
  tp.vt_count = pl.vtiles;
  tp.scale2 = pp.scale2;
  tp.rows = static_cast<long long>(crows);
  tp.partials = reinterpret_cast<float2*>(ws + pl.off_partials);
  tp.zlabel = reinterpret_cast<float*>(ws + pl.off_zlabel);
  tp.lse2 = reinterpret_cast<float*>(ws + pl.off_lse2);
  tp.status = status;
  int slots = 0;
  const int rows_smem = 2 * ce_rows_cfg::kTokens * a->d;
  if (a->T <= ce_rows_cfg::kTokens && rows_smem <= ce_rows_cfg::kMaxTokenBytes) {
    CeRowsParams rp{};
    rp.V = a->V;
    rp.d = a->d;
    rp.plan = pp.plan;
    rp.cy = pp.cy;
    rp.hc = hc;
    rp.weight = pp.head;
    rp.ldw = a->ldw;
    rp.rows = tp.rows;
    rp.scale2 = tp.scale2;
    rp.partials = tp.partials;
    rp.zlabel = tp.zlabel;
    // Batches of loads that divide a warp's share of K waste none: 3 steps where the share is a multiple of 3 and not of
    // 4 (d = 1536: 6), else 4.  Smaller batches leave registers for a third block per SM.
    const int share = (a->d / 32 + ce_rows_cfg::kWarps - 1) / ce_rows_cfg::kWarps;
    const bool three = share % 3 == 0 && share % 4 != 0 && rows_smem <= 48 * 1024;
    // as many blocks as are resident, as far as there are groups of 16 rows (the workspace has room for three per SM)
    slots = std::max(1, std::min({(three ? 3 : 2) * di.sms, (a->V + 15) / 16}));
    auto k = three ? ce_rows_kernel<3> : ce_rows_kernel<4>;
    if (set_smem(k, ce_rows_cfg::kMaxTokenBytes) != NPD_OK) return NPD_ECUDA;
    const cudaError_t e = launch_ex(k, slots, ce_rows_cfg::kThreads, rows_smem, st, pdl, rp);
    ++g_launches;
    if (e != cudaSuccess) return NPD_ECUDA;
  } else if ((rc = launch_pair_tile<CeForwardEpi>(mh, mw, tp, pl.clusters, st, pdl)) != NPD_OK) {
    return rc;
  }

  CeMergeParams mp{};
  mp.T = a->T;
  mp.slots = slots;
  mp.plan = pp.plan;
  mp.cidx = pp.cidx;
  mp.partials = tp.partials;
  mp.rows = tp.rows;
  mp.zlabel = tp.zlabel;
  mp.zy = pp.zy;
  mp.nll = a->nll;
  mp.lse = a->lse;
  mp.lse2 = reinterpret_cast<float*>(ws + pl.off_lse2);
  if ((slots > 0 ? launch_ex(ce_merge_rows_kernel, a->T, 256, 0, st, pdl, mp)
                 : launch_ex(ce_merge_kernel, (a->T + 31) / 32, 256, 0, st, pdl, mp)) != cudaSuccess)
    return NPD_ECUDA;
  ++g_launches;
  if (!pl.grads) return NPD_OK;

  const float scale = a->grad_scale / a->temperature;
  __nv_bfloat16* gbuf = reinterpret_cast<__nv_bfloat16*>(ws + pl.off_g);
  const bool wf32 = a->d_weight_dtype == NPD_DTYPE_F32;
  for (int c = 0; c < pl.nchunks; ++c) {
    const int col0 = c * pl.chunk_cols;
    const int cols = std::min(pl.chunk_cols, a->V - col0);
    if (cols <= 0) break;
    const int cols_pad = std::min(pl.chunk_cols, pl.vtiles * 256 - col0);
    CeTileParams gp = tp;
    gp.vt_begin = col0 / 256;
    gp.vt_count = cols_pad / 256;
    gp.gbuf = gbuf;
    gp.ldg = pl.chunk_cols;
    gp.g_col0 = col0;
    if ((rc = launch_pair_tile<CeGradientEpi>(mh, mw, gp, pl.clusters, st, pdl)) != NPD_OK) return rc;

    GemmProblem pr[2] = {};
    GemmOperands ops[2] = {};
    chunk_problems(a->d, cols, wf32, (a->flags & NPD_CE_ACCUMULATE_DW) != 0, pr);
    pr[0].alpha = scale;  // dW rows; dH is scaled when its sums are converted
    void* dw_rows = a->d_weight == nullptr ? nullptr
                    : wf32 ? static_cast<void*>(static_cast<float*>(a->d_weight) + static_cast<size_t>(col0) * a->ld_dw)
                           : static_cast<void*>(static_cast<__nv_bfloat16*>(a->d_weight) + static_cast<size_t>(col0) * a->ld_dw);
    ops[0] = {gbuf, pl.chunk_cols, hc, a->d, dw_rows, a->ld_dw};
    const __nv_bfloat16* w_rows = static_cast<const __nv_bfloat16*>(a->weight) + static_cast<size_t>(col0) * a->ldw;
    ops[1] = {gbuf, pl.chunk_cols, w_rows, a->ldw, dh_acc, a->d};
    if (a->d_weight == nullptr) {
      pr[0].M = 0;  // a frozen head: only the second product
      ops[0] = ops[1];
    }
    if ((rc = launch_gemm(a->d_hidden != nullptr ? 2 : 1, pr, ops, pp.plan, pl.row_blocks, status, di.sms, st, pdl)) != NPD_OK)
      return rc;
  }
  if (a->d_hidden != nullptr) {
    const long long n = static_cast<long long>(a->T) * (a->d / 8);
    if (launch_ex(ce_scatter_kernel, static_cast<int>((n + 255) / 256), 256, 0, st, pdl, dh_acc, pp.cidx, a->T, a->d, scale,
                  static_cast<__nv_bfloat16*>(a->d_hidden), a->ld_dh) != cudaSuccess)
      return NPD_ECUDA;
    ++g_launches;
  }
  return NPD_OK;
}

}  // extern "C"
