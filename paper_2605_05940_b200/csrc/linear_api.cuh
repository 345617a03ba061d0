// Host side of npd_linear_fwd / npd_linear_bwd.  Included by npd_api.cu, whose helpers it uses.
#pragma once

#include "linear_kernels.cuh"

namespace {

int check_linear(const npd_linear_args* a, bool backward, bool need_pointers) {
  if (a == nullptr || a->size != sizeof(npd_linear_args)) return NPD_EINVAL;
  if (a->M < 1 || a->N < 1 || a->K < 1) return NPD_EINVAL;
  if (a->activation < NPD_ACT_NONE || a->activation > NPD_ACT_SILU) return NPD_EINVAL;
  if (a->bias_dtype != NPD_DTYPE_BF16 && a->bias_dtype != NPD_DTYPE_F32) return NPD_EINVAL;
  if (a->y_dtype != NPD_DTYPE_BF16 && a->y_dtype != NPD_DTYPE_F32) return NPD_EINVAL;
  if (a->dw_dtype != NPD_DTYPE_BF16 && a->dw_dtype != NPD_DTYPE_F32) return NPD_EINVAL;
  if (a->flags & ~NPD_LINEAR_ACCUMULATE_DW) return NPD_EINVAL;
  if ((a->flags & NPD_LINEAR_ACCUMULATE_DW) && a->dw_dtype != NPD_DTYPE_F32) return NPD_EINVAL;
  // extents and numbers of tiles are 32-bit: a product of 2^46 is at most 2^30 + (2^30 + 2^30) / 256 + 1 tiles
  if (a->M > (1 << 30) || a->N > (1 << 30) || a->K > (1 << 30)) return NPD_ESHAPE;
  const long long M = a->M, N = a->N, K = a->K;
  if (std::max({M * N, M * K, N * K}) > 1ll << 46) return NPD_ESHAPE;
  if (!need_pointers) return NPD_OK;
  const long long ye = a->y_dtype == NPD_DTYPE_F32 ? 4 : 2, we = a->dw_dtype == NPD_DTYPE_F32 ? 4 : 2,
                  be = a->bias_dtype == NPD_DTYPE_F32 ? 4 : 2;
  struct M_ { const void* p; int64_t ld; long long cols, es; };
  auto strided = [&](std::initializer_list<M_> ms) {
    for (const M_& m : ms) {
      if (m.p == nullptr) continue;
      if (m.ld < m.cols) return static_cast<int>(NPD_ESHAPE);
      if ((m.ld * m.es) % 16 || !aligned16(m.p)) return static_cast<int>(NPD_EALIGN);
    }
    return static_cast<int>(NPD_OK);
  };
  auto ext = [](const void* p, long long rows, long long cols, long long ld, long long es) {
    return Extent{p, rows, cols * es, ld * es};
  };
  const Extent x = ext(a->x, M, K, a->ldx, 2), w = ext(a->weight, N, K, a->ldw, 2);
  const Extent z = ext(a->preact, M, N, a->ldz, 2);
  if (a->weight == nullptr) return NPD_EINVAL;
  int rc;
  if (!backward) {
    if (a->x == nullptr || a->y == nullptr) return NPD_EINVAL;
    if ((rc = strided({{a->x, a->ldx, K, 2}, {a->weight, a->ldw, K, 2}, {a->y, a->ldy, N, ye}, {a->residual, a->ldr, N, ye},
                       {a->preact, a->ldz, N, 2}})) != NPD_OK)
      return rc;
    if (reinterpret_cast<uintptr_t>(a->bias) & (be - 1)) return NPD_EALIGN;
    if (reinterpret_cast<uintptr_t>(a->status) & 3) return NPD_EALIGN;
    const Extent y = ext(a->y, M, N, a->ldy, ye), res = ext(a->residual, M, N, a->ldr, ye), bias{a->bias, 1, N * be, N * be};
    if (bad_overlap(y, res, true) || extents_touch(z, res)) return NPD_EINVAL;
    for (const Extent* o : {&y, &z})
      for (const Extent* in : {&x, &w, &bias})
        if (extents_touch(*o, *in)) return NPD_EINVAL;
    return extents_touch(y, z) ? NPD_EINVAL : NPD_OK;
  }
  if (a->dy == nullptr || (a->dx == nullptr && a->dw == nullptr && a->dbias == nullptr)) return NPD_EINVAL;
  if (a->activation != NPD_ACT_NONE && a->preact == nullptr) return NPD_EINVAL;
  if (a->dw != nullptr && a->x == nullptr) return NPD_EINVAL;
  if ((rc = strided({{a->weight, a->ldw, K, 2}, {a->dy, a->lddy, N, 2}, {a->preact, a->ldz, N, 2}, {a->dx, a->lddx, K, 2},
                     {a->dw, a->lddw, K, we}})) != NPD_OK)
    return rc;
  if (a->dw != nullptr && (rc = strided({{a->x, a->ldx, K, 2}})) != NPD_OK) return rc;
  if (reinterpret_cast<uintptr_t>(a->dbias) & 3) return NPD_EALIGN;
  const Extent dy = ext(a->dy, M, N, a->lddy, 2), dx = ext(a->dx, M, K, a->lddx, 2), dw = ext(a->dw, N, K, a->lddw, we),
               db{a->dbias, 1, 4 * N, 4 * N};
  const Extent x_read = a->dw != nullptr ? x : Extent{nullptr, 0, 0, 0};
  const Extent z_read = a->activation != NPD_ACT_NONE ? z : Extent{nullptr, 0, 0, 0};
  for (const Extent* o : {&dx, &dw, &db})
    for (const Extent* in : {&dy, &x_read, &w, &z_read})
      if (extents_touch(*o, *in)) return NPD_EINVAL;
  return extents_touch(dx, dw) || extents_touch(dx, db) || extents_touch(dw, db) ? NPD_EINVAL : NPD_OK;
}

struct LinearPlan {
  int row_blocks, rows_per_block;  // of the dz kernel
  long long lddz;
  size_t off_part, total;
};

LinearPlan linear_plan(const npd_linear_args* a, int sms) {
  LinearPlan pl{};
  const int across = (a->N + 255) / 256;
  // about eight blocks of 256 threads per SM; at least 8 rows (one per warp) each
  const int want = std::max(1, 8 * sms / across);
  pl.rows_per_block = std::max(8, (a->M + want - 1) / want);
  pl.row_blocks = (a->M + pl.rows_per_block - 1) / pl.rows_per_block;
  pl.lddz = (static_cast<long long>(a->N) + 7) / 8 * 8;
  size_t off = 1024;  // status word first, as in the other workspaces
  if (a->activation != NPD_ACT_NONE) off = align_up(off + 2 * static_cast<size_t>(a->M) * pl.lddz, 1024);
  pl.off_part = off;
  off = align_up(off + sizeof(float) * static_cast<size_t>(pl.row_blocks) * pl.lddz, 1024);
  pl.total = off;
  return pl;
}

template <bool kRagged>
void (*linear_dz_pick(int act))(LinearGradParams) {
  switch (act) {
    case NPD_ACT_RELU: return linear_dz_kernel<kActRelu, kRagged>;
    case NPD_ACT_GELU: return linear_dz_kernel<kActGelu, kRagged>;
    case NPD_ACT_GELU_TANH: return linear_dz_kernel<kActGeluTanh, kRagged>;
    case NPD_ACT_SILU: return linear_dz_kernel<kActSilu, kRagged>;
    default: return linear_dz_kernel<kActNone, kRagged>;
  }
}

template <int kG>
cudaError_t launch_rows(const LinearParams& p, cudaStream_t st) {
  return launch_ex(linear_rows_kernel<kG>, (p.N + 15) / 16, 32 * rows_cfg::kWarps, 0, st, false, p);
}

template <bool kY32, bool kKeepZ, int kBN>
int launch_linear_tiles_n(const npd_linear_args* a, LinearParams p, int sms, cudaStream_t st) {
  CUtensorMap mx, mw;
  if (!make_map(&mx, a->x, a->K, a->M, a->ldx, 64, 128) || !make_map(&mw, a->weight, a->K, a->N, a->ldw, 64, kBN / 2))
    return NPD_ECUDA;
  p.ntiles = (a->N + kBN - 1) / kBN;
  const int pairs = std::max(1, std::min(p.mtiles * p.ntiles, sms / 2));
  return launch_pair_tile<LinearEpi<kY32, kKeepZ, kBN>>(mx, mw, p, pairs, st, false);
}

// Width of the tiles: the narrowest whose number still fits one round of the CTA pairs, so that a small problem
// spreads over more of them, else 256 (a wide tile feeds the tensor cores better).  Measured at K = 4096, N = 4096, 256 /
// 128 / 64 wide: M = 256 32.1 / 25.0 / 23.9 us (16, 32, 64 tiles), M = 512 32.8 / 26.0 / 40.8, M = 1024 34.1 / 43.8 / 74.4.
int linear_tile_width(int M, int N, int pairs) {
  const long long rows = (M + 255) / 256;
  for (int bn : {64, 128})
    if (rows * ((N + bn - 1) / bn) <= pairs) return bn;
  return 256;
}

template <bool kY32, bool kKeepZ>
int launch_linear_tiles(const npd_linear_args* a, const LinearParams& p, int sms, cudaStream_t st) {
  const int bn = linear_tile_width(a->M, a->N, std::max(1, sms / 2));
  if (bn == 256) return launch_linear_tiles_n<kY32, kKeepZ, 256>(a, p, sms, st);
  if (bn == 128) return launch_linear_tiles_n<kY32, kKeepZ, 128>(a, p, sms, st);
  return launch_linear_tiles_n<kY32, kKeepZ, 64>(a, p, sms, st);
}
}  // namespace

extern "C" {

int npd_linear_fwd(const npd_linear_args* a, void* cuda_stream) {
  g_launches = 0;
  int rc = check_linear(a, false, true);
  if (rc != NPD_OK) return rc;
  DeviceInfo di;
  if ((rc = device_info(&di)) != NPD_OK) return rc;
  if (di.cc_major != 10) return NPD_EARCH;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  LinearParams p{};
  p.M = a->M;
  p.N = a->N;
  p.K = a->K;
  p.ksteps = (a->K + 63) / 64;
  p.act = a->activation;
  p.x = static_cast<const __nv_bfloat16*>(a->x);
  p.w = static_cast<const __nv_bfloat16*>(a->weight);
  p.ldx = a->ldx;
  p.ldw = a->ldw;
  p.bias = a->bias;
  p.bias_f32 = a->bias_dtype == NPD_DTYPE_F32;
  p.residual = a->residual;
  p.ldr = a->ldr;
  p.y = a->y;
  p.z = static_cast<__nv_bfloat16*>(a->preact);
  p.ldy = a->ldy;
  p.ldz = a->ldz;
  p.y_f32 = a->y_dtype == NPD_DTYPE_F32;
  // whole 32-byte sectors per store where the rows allow it
  const int ye = p.y_f32 ? 4 : 2;
  p.wide_y = reinterpret_cast<uintptr_t>(a->y) % 32 == 0 && a->ldy * ye % 32 == 0;
  p.wide_z = reinterpret_cast<uintptr_t>(a->preact) % 32 == 0 && a->ldz * 2 % 32 == 0;
  p.status = a->status;
  if (a->M <= rows_cfg::kRowsMax) {
    const cudaError_t e = a->M <= 8    ? launch_rows<1>(p, st)
                          : a->M <= 16 ? launch_rows<2>(p, st)
                                       : launch_rows<4>(p, st);
    ++g_launches;
    return e == cudaSuccess ? NPD_OK : NPD_ECUDA;
  }
  p.mtiles = (a->M + 255) / 256;
  p.group = static_cast<int>(std::min<long long>(p.mtiles, std::max<long long>(4, (32ll << 20) / (512ll * a->K))));
  if (p.y_f32)
    return p.z != nullptr ? launch_linear_tiles<true, true>(a, p, di.sms, st) : launch_linear_tiles<true, false>(a, p, di.sms, st);
  return p.z != nullptr ? launch_linear_tiles<false, true>(a, p, di.sms, st) : launch_linear_tiles<false, false>(a, p, di.sms, st);
}

int npd_linear_workspace_bytes(const npd_linear_args* args, size_t* out_bytes) {
  if (out_bytes == nullptr) return NPD_EINVAL;
  int rc = check_linear(args, true, false);
  if (rc != NPD_OK) return rc;
  DeviceInfo di;
  if ((rc = device_info(&di)) != NPD_OK) return rc;
  *out_bytes = linear_plan(args, di.sms).total;
  return NPD_OK;
}

int npd_linear_bwd(const npd_linear_args* a, void* cuda_stream) {
  g_launches = 0;
  int rc = check_linear(a, true, true);
  if (rc != NPD_OK) return rc;
  DeviceInfo di;
  if ((rc = device_info(&di)) != NPD_OK) return rc;
  if (di.cc_major != 10) return NPD_EARCH;
  const LinearPlan pl = linear_plan(a, di.sms);
  if (a->workspace == nullptr || (reinterpret_cast<uintptr_t>(a->workspace) & 1023u) || a->workspace_bytes < pl.total)
    return NPD_EWORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  uint8_t* ws = static_cast<uint8_t*>(a->workspace);
  int* status = reinterpret_cast<int*>(ws);
  if (cudaMemsetAsync(status, 0, sizeof(int), st) != cudaSuccess) return NPD_ECUDA;
  const bool act = a->activation != NPD_ACT_NONE, products = a->dx != nullptr || a->dw != nullptr;
  const void* dz = a->dy;
  long long lddz = a->lddy;
  if ((act && products) || a->dbias != nullptr) {
    LinearGradParams gp{};
    gp.M = a->M;
    gp.N = a->N;
    gp.act = a->activation;
    gp.rows_per_block = pl.rows_per_block;
    gp.dy = static_cast<const __nv_bfloat16*>(a->dy);
    gp.z = static_cast<const __nv_bfloat16*>(a->preact);
    gp.dz = reinterpret_cast<__nv_bfloat16*>(ws + 1024);
    gp.lddy = a->lddy;
    gp.ldz = a->ldz;
    gp.lddz = pl.lddz;
    gp.ldpart = pl.lddz;  // a multiple of 8
    gp.part = a->dbias != nullptr ? reinterpret_cast<float*>(ws + pl.off_part) : nullptr;
    if (act) {
      dz = gp.dz;
      lddz = pl.lddz;
    }
    const auto k = a->N % 8 != 0 ? linear_dz_pick<true>(a->activation) : linear_dz_pick<false>(a->activation);
    cudaError_t e = launch_dim(k, dim3(static_cast<unsigned>((a->N + 255) / 256), static_cast<unsigned>(pl.row_blocks)), 256, 0, st,
                               false, gp);
    ++g_launches;
    if (e == cudaSuccess && a->dbias != nullptr) {
      e = launch_dim(column_sum_kernel, dim3(static_cast<unsigned>((a->N + 31) / 32)), 1024, 0, st, true, gp.part, pl.row_blocks,
                     gp.ldpart, a->N, a->dbias);
      ++g_launches;
    }
    if (e != cudaSuccess) return NPD_ECUDA;
  }
  if (!products) return NPD_OK;
  GemmProblem pr[2] = {};
  GemmOperands ops[2] = {};
  // dW[n,k] = sum_m dz[m,n] x[m,k]
  GemmProblem gw{};
  gw.M = a->N;
  gw.N = a->K;
  gw.K = a->M;
  gw.a_mn = gw.b_mn = 1;
  gw.k_splits = 1;
  gw.out_f32 = a->dw_dtype == NPD_DTYPE_F32;
  gw.out_reduce = (a->flags & NPD_LINEAR_ACCUMULATE_DW) ? 1 : 0;
  const GemmOperands ow{dz, lddz, a->x, a->ldx, a->dw, a->lddw};
  // dx[m,k] = sum_n dz[m,n] W[n,k]
  GemmProblem gx{};
  gx.M = a->M;
  gx.N = a->K;
  gx.K = a->N;
  gx.b_mn = 1;
  gx.k_splits = 1;
  const GemmOperands ox{dz, lddz, a->weight, a->ldw, a->dx, a->lddx};
  int n = 0;
  if (a->dw != nullptr) {
    pr[n] = gw;
    ops[n++] = ow;
  }
  if (a->dx != nullptr) {
    pr[n] = gx;
    ops[n++] = ox;
  }
  return launch_gemm(n, pr, ops, nullptr, 0, status, di.sms, st, true, true);
}

}  // extern "C"
