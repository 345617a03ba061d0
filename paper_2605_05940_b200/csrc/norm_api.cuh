// Host side of npd_norm_fwd / npd_norm_bwd.  Included by npd_api.cu, whose helpers it uses.
#pragma once

#include "norm_kernels.cuh"

namespace {

// A row-major matrix as a byte pattern: `rows` rows of `width` bytes, `stride` bytes apart.
struct Extent {
  const void* p;
  long long rows, width, stride;
};
// Whether two matrices share a byte.  Column windows of one wider buffer (equal strides) may
// interleave without touching.
bool extents_touch(const Extent& a, const Extent& b) {
  if (a.p == nullptr || b.p == nullptr || a.rows < 1 || b.rows < 1 || a.width < 1 || b.width < 1) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  const uintptr_t a1 = a0 + static_cast<uintptr_t>((a.rows - 1) * a.stride + a.width);
  const uintptr_t b1 = b0 + static_cast<uintptr_t>((b.rows - 1) * b.stride + b.width);
  if (a1 <= b0 || b1 <= a0) return false;
  if (a.stride != b.stride || a.stride < a.width || b.stride < b.width) return true;
  const long long s = a.stride;
  const long long delta = static_cast<long long>((b0 >= a0 ? b0 - a0 : static_cast<uintptr_t>(s) - (a0 - b0) % s) % s);
  return delta < a.width || s - delta < b.width;
}
// The very same matrix: a result may take its operand's place element by element.
bool extents_same(const Extent& a, const Extent& b) {
  return a.p != nullptr && a.p == b.p && a.rows == b.rows && a.width == b.width && a.stride == b.stride;
}
// An output that has to lie apart from an operand, `in_place` = may be exactly that operand.
bool bad_overlap(const Extent& out, const Extent& in, bool in_place) {
  return extents_touch(out, in) && !(in_place && extents_same(out, in));
}

struct NormPlan {
  int vec, threads, span, smem, grid, part_d;
  bool narrow;
  size_t ws;
};

NormPlan norm_plan(const npd_norm_args* a, int sms, bool backward) {
  using namespace norm_cfg;
  NormPlan pl{};
  pl.vec = a->d <= (backward ? kMaxSmallBwd : kMaxSmallFwd) ? 1 : (a->d <= kMaxSmallFwd ? 2 : 4);
  const int per = 8 * pl.vec;
  pl.narrow = a->d <= kNarrowD;
  pl.threads = pl.narrow ? kNarrowThreads : ((a->d + per - 1) / per + 31) / 32 * 32;
  pl.span = a->d <= 64 ? 8 : (a->d <= 128 ? 16 : 32);
  const int rows = pl.narrow ? pl.threads / pl.span : 1;  // of a CTA at a time
  // sums over rows (and gains up to kMaxSmallFwd), or where the warps' sums meet
  pl.smem = !backward ? 0 : pl.vec > 1 ? 64 * pl.vec * pl.threads * (pl.vec == 2 ? 2 : 1) : pl.narrow ? 2 * pl.threads * pl.span : 0;
  // Resident CTAs per SM, by threads and (an estimate of) registers: every CTA goes through its share
  // of the rows.  Several per SM, so that one CTA's barriers run under another one's loads.
  int per_sm = (backward || pl.vec > 1 ? 512 : 1024) / pl.threads;
  per_sm = std::max(1, std::min(per_sm, 16));
  pl.grid = std::min((a->T + rows - 1) / rows, sms * per_sm);
  pl.part_d = (a->d + 3) / 4 * 4;
  pl.ws = align_up(sizeof(float) * 2 * static_cast<size_t>(pl.part_d) * pl.grid, 1024);
  return pl;
}

int check_norm(const npd_norm_args* a, bool backward, bool need_pointers) {
  if (a == nullptr || a->size != sizeof(npd_norm_args)) return NPD_EINVAL;
  if (a->T < 1 || a->d < 1) return NPD_EINVAL;
  if (a->d > norm_cfg::kMaxD || a->T > (1 << 30)) return NPD_ESHAPE;
  if (a->stream_dtype != NPD_DTYPE_BF16 && a->stream_dtype != NPD_DTYPE_F32) return NPD_EINVAL;
  if (a->weight_dtype != NPD_DTYPE_BF16 && a->weight_dtype != NPD_DTYPE_F32) return NPD_EINVAL;
  if (a->flags & ~NPD_NORM_POST) return NPD_EINVAL;
  if (!(a->eps >= 0.f) || !std::isfinite(a->eps) || !std::isfinite(a->weight_offset) ||
      !std::isfinite(a->residual_scale) || !std::isfinite(a->branch_scale))
    return NPD_EINVAL;
  if (!need_pointers) return NPD_OK;
  const bool sf = a->stream_dtype == NPD_DTYPE_F32;
  const long long es = sf ? 4 : 2, T = a->T, d = a->d;
  // {pointer, row stride, element size, may have row stride 0}
  struct M { const void* p; int64_t ld; long long es; bool bcast; };
  const M mats[] = {{a->x, a->ldx, 2, false}, {a->residual, a->ldr, es, false}, {a->gate, a->ldg, 2, true},
                    {a->h, a->ldh, es, false}, {a->y, a->ldy, 2, false}, {a->dy, a->lddy, 2, false},
                    {a->dh, a->lddh, es, false}, {a->dx, a->lddx, 2, false}, {a->dresidual, a->lddr, es, false}};
  for (const M& m : mats) {
    if (m.p == nullptr) continue;
    if (m.ld < (m.bcast && m.ld == 0 ? 0 : d)) return NPD_ESHAPE;
    if ((m.ld * m.es) % 16 || !aligned16(m.p)) return NPD_EALIGN;
  }
  if ((a->flags & NPD_NORM_POST) && a->x == nullptr) return NPD_EINVAL;
  if (a->gate != nullptr && a->x == nullptr) return NPD_EINVAL;
  const uintptr_t wmask = a->weight_dtype == NPD_DTYPE_F32 ? 3 : 1;
  if ((reinterpret_cast<uintptr_t>(a->post_weight) & wmask) || (reinterpret_cast<uintptr_t>(a->pre_weight) & wmask))
    return NPD_EALIGN;
  const long long wb = a->weight_dtype == NPD_DTYPE_F32 ? 4 : 2;
  auto ext = [&](const void* p, int64_t ld, long long e) { return Extent{p, T, d * e, ld * e}; };
  const Extent x = ext(a->x, a->ldx, 2), res = ext(a->residual, a->ldr, es), h = ext(a->h, a->ldh, es),
               y = ext(a->y, a->ldy, 2), dy = ext(a->dy, a->lddy, 2), dh = ext(a->dh, a->lddh, es),
               dx = ext(a->dx, a->lddx, 2), dr = ext(a->dresidual, a->lddr, es);
  const Extent gate = a->ldg == 0 ? Extent{a->gate, 1, 2 * d, 2 * d} : ext(a->gate, a->ldg, 2);
  const Extent wp{a->post_weight, 1, wb * d, wb * d}, wq{a->pre_weight, 1, wb * d, wb * d};
  if (!backward) {
    if (a->x == nullptr && a->residual == nullptr) return NPD_EINVAL;
    if (a->h == nullptr && a->y == nullptr) return NPD_EINVAL;
    for (const Extent* o : {&h, &y}) {
      for (const Extent* in : {&x, &res})
        if (bad_overlap(*o, *in, true)) return NPD_EINVAL;
      for (const Extent* in : {&gate, &wp, &wq})
        if (bad_overlap(*o, *in, false)) return NPD_EINVAL;
    }
    return extents_touch(h, y) ? NPD_EINVAL : NPD_OK;
  }
  if (a->dy == nullptr && a->dh == nullptr) return NPD_EINVAL;
  if (a->dy != nullptr && a->h == nullptr) return NPD_EINVAL;
  if (a->dx != nullptr && a->x == nullptr && (a->flags & NPD_NORM_POST)) return NPD_EINVAL;
  if (a->d_post_weight != nullptr && !(a->flags & NPD_NORM_POST)) return NPD_EINVAL;
  if (a->d_pre_weight != nullptr && a->dy == nullptr) return NPD_EINVAL;
  if (a->d_gate != nullptr && a->gate == nullptr) return NPD_EINVAL;
  if (a->dx == nullptr && a->dresidual == nullptr && a->d_post_weight == nullptr && a->d_pre_weight == nullptr &&
      a->d_gate == nullptr)
    return NPD_EINVAL;
  Extent dg{nullptr, 0, 0, 0};
  if (a->d_gate != nullptr) {
    if (a->ldg == 0) {
      if (reinterpret_cast<uintptr_t>(a->d_gate) & 3) return NPD_EALIGN;
      dg = Extent{a->d_gate, 1, 4 * d, 4 * d};
    } else {
      if (a->lddg < d) return NPD_ESHAPE;
      if (a->lddg % 8 || !aligned16(a->d_gate)) return NPD_EALIGN;
      dg = ext(a->d_gate, a->lddg, 2);
    }
  }
  if ((reinterpret_cast<uintptr_t>(a->d_post_weight) & 3) || (reinterpret_cast<uintptr_t>(a->d_pre_weight) & 3))
    return NPD_EALIGN;
  const Extent gp{a->d_post_weight, 1, 4 * d, 4 * d}, gq{a->d_pre_weight, 1, 4 * d, 4 * d};
  const Extent outs[] = {dx, dr, dg, gp, gq}, ins[] = {dy, h, dh, x, gate, wp, wq};
  for (int o = 0; o < 5; ++o) {
    for (int i = 0; i < 7; ++i)
      // dx, dresidual and a per-token gate gradient may take the place of a per-row operand
      if (bad_overlap(outs[o], ins[i], o < 2 || (o == 2 && a->ldg != 0)) ||
          (extents_same(outs[o], ins[i]) && i >= 4 && !(i == 4 && a->ldg != 0 && o <= 2)))
        return NPD_EINVAL;
    for (int q = o + 1; q < 5; ++q)
      if (extents_touch(outs[o], outs[q])) return NPD_EINVAL;
  }
  return NPD_OK;
}

NormParams norm_params(const npd_norm_args* a, const NormPlan& pl, bool backward) {
  NormParams p{};
  p.span = pl.span;
  p.T = a->T;
  p.d = a->d;
  p.x = static_cast<const __nv_bfloat16*>(a->x);
  p.residual = a->residual;
  p.gate = static_cast<const __nv_bfloat16*>(a->gate);
  p.post = (a->flags & NPD_NORM_POST) ? 1 : 0;
  p.w_post = p.post ? a->post_weight : nullptr;
  p.w_pre = (backward ? a->dy != nullptr : a->y != nullptr) ? a->pre_weight : nullptr;
  p.w_f32 = a->weight_dtype == NPD_DTYPE_F32;
  p.ldx = a->ldx;
  p.ldr = a->ldr;
  p.ldg = a->ldg;
  p.eps = a->eps;
  p.offset = a->weight_offset;
  p.res_scale = a->residual_scale;
  p.branch_scale = a->branch_scale;
  p.h = a->h;
  p.y = static_cast<__nv_bfloat16*>(a->y);
  p.ldh = a->ldh;
  p.ldy = a->ldy;
  if (backward) {
    p.dy = static_cast<const __nv_bfloat16*>(a->dy);
    p.dh = a->dh;
    p.dx = static_cast<__nv_bfloat16*>(a->dx);
    p.dres = a->dresidual;
    p.dgate = a->gate != nullptr && a->ldg != 0 ? static_cast<__nv_bfloat16*>(a->d_gate) : nullptr;
    p.lddy = a->lddy;
    p.lddh = a->lddh;
    p.lddx = a->lddx;
    p.lddres = a->lddr;
    p.lddgate = a->lddg;
    p.want = (a->d_pre_weight != nullptr ? 1 : 0) | (a->d_post_weight != nullptr ? 2 : 0) |
             (a->d_gate != nullptr && a->ldg == 0 ? 4 : 0);
  }
  return p;
}

using NormKernel = void (*)(NormParams);

// The instances by size of the block, and what the call has (see the kernels).
template <bool kF32, bool kGate, bool kRagged>
NormKernel norm_fwd_pick(const NormPlan& pl) {
  if (pl.narrow) return norm_fwd_kernel<kF32, 1, norm_cfg::kNarrowThreads, kGate, kRagged, true>;
  return pl.threads <= 512 ? norm_fwd_kernel<kF32, 1, 512, kGate, kRagged, false>
                           : norm_fwd_kernel<kF32, 1, 1024, kGate, kRagged, false>;
}
template <bool kF32>
NormKernel norm_fwd_pick(const NormPlan& pl, bool token_gate, bool ragged) {
  if (pl.vec > 1) return norm_fwd_kernel<kF32, 4, 512, true, true, false>;
  if (token_gate) return ragged ? norm_fwd_pick<kF32, true, true>(pl) : norm_fwd_pick<kF32, true, false>(pl);
  return ragged ? norm_fwd_pick<kF32, false, true>(pl) : norm_fwd_pick<kF32, false, false>(pl);
}
template <bool kF32, int kForm, bool kGate>
NormKernel norm_bwd_pick(const NormPlan& pl) {
  if (pl.narrow) return norm_bwd_kernel<kF32, 1, kForm, kGate, norm_cfg::kNarrowThreads, true>;
  return pl.threads <= 256 ? norm_bwd_kernel<kF32, 1, kForm, kGate, 256, false> : norm_bwd_kernel<kF32, 1, kForm, kGate, 512, false>;
}
template <bool kF32>
NormKernel norm_bwd_pick(const NormPlan& pl, int form, bool token_gate) {
  if (pl.vec > 1 && form < 2) return pl.vec == 2 ? norm_bwd_kernel<kF32, 2, 0, false, 512, false> : norm_bwd_kernel<kF32, 4, 0, false, 512, false>;
  if (pl.vec == 2) return token_gate ? norm_bwd_kernel<kF32, 2, 2, true, 512, false> : norm_bwd_kernel<kF32, 2, 2, false, 512, false>;
  if (pl.vec == 4) return token_gate ? norm_bwd_kernel<kF32, 4, 2, true, 512, false> : norm_bwd_kernel<kF32, 4, 2, false, 512, false>;
  if (form == 0) return norm_bwd_pick<kF32, 0, false>(pl);
  if (token_gate) return form == 1 ? norm_bwd_pick<kF32, 1, true>(pl) : norm_bwd_pick<kF32, 2, true>(pl);
  return form == 1 ? norm_bwd_pick<kF32, 1, false>(pl) : form == 2 ? norm_bwd_pick<kF32, 2, false>(pl) : norm_bwd_pick<kF32, 3, false>(pl);
}

}  // namespace

extern "C" {

int npd_norm_workspace_bytes(const npd_norm_args* args, size_t* out_bytes) {
  if (out_bytes == nullptr) return NPD_EINVAL;
  int rc = check_norm(args, true, false);
  if (rc != NPD_OK) return rc;
  DeviceInfo di;
  if ((rc = device_info(&di)) != NPD_OK) return rc;
  *out_bytes = norm_plan(args, di.sms, true).ws;
  return NPD_OK;
}

int npd_norm_fwd(const npd_norm_args* a, void* cuda_stream) {
  g_launches = 0;
  int rc = check_norm(a, false, true);
  if (rc != NPD_OK) return rc;
  DeviceInfo di;
  if ((rc = device_info(&di)) != NPD_OK) return rc;
  if (di.cc_major != 10) return NPD_EARCH;
  const NormPlan pl = norm_plan(a, di.sms, false);
  const bool sf = a->stream_dtype == NPD_DTYPE_F32;
  const bool token_gate = a->gate != nullptr && a->ldg != 0, ragged = a->d % 8 != 0;
  const NormKernel k = sf ? norm_fwd_pick<true>(pl, token_gate, ragged) : norm_fwd_pick<false>(pl, token_gate, ragged);
  const cudaError_t e = launch_ex(k, pl.grid, pl.threads, 0, static_cast<cudaStream_t>(cuda_stream), false,
                                  norm_params(a, pl, false));
  ++g_launches;
  return e == cudaSuccess ? NPD_OK : NPD_ECUDA;
}

int npd_norm_bwd(const npd_norm_args* a, void* cuda_stream) {
  g_launches = 0;
  int rc = check_norm(a, true, true);
  if (rc != NPD_OK) return rc;
  DeviceInfo di;
  if ((rc = device_info(&di)) != NPD_OK) return rc;
  if (di.cc_major != 10) return NPD_EARCH;
  const NormPlan pl = norm_plan(a, di.sms, true);
  NormParams p = norm_params(a, pl, true);
  p.part_d = pl.part_d;
  if (p.want != 0) {
    if (a->workspace == nullptr || (reinterpret_cast<uintptr_t>(a->workspace) & 15u) || a->workspace_bytes < pl.ws)
      return NPD_EWORKSPACE;
    p.part = static_cast<float*>(a->workspace);
  }
  const bool sf = a->stream_dtype == NPD_DTYPE_F32;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool token_gate = p.gate != nullptr && p.ldg != 0;
  const bool full = p.dy != nullptr && p.dh != nullptr && p.x != nullptr && p.dx != nullptr && p.dres != nullptr &&
                    (!token_gate || p.dgate != nullptr);
  const int form = !full ? 0 : a->d % 8 != 0 ? 1 : a->d % 256 != 0 || token_gate ? 2 : 3;
  const NormKernel k = sf ? norm_bwd_pick<true>(pl, form, token_gate) : norm_bwd_pick<false>(pl, form, token_gate);
  const int ring = pl.vec == 1 && full && !sf ? norm_cfg::kRing * pl.threads * 16 * (token_gate ? 5 : 4) : 0;
  const int smem = std::max(ring, pl.smem);
  if (smem > 0 && set_smem(k, norm_cfg::kMaxSmem) != NPD_OK) return NPD_ECUDA;
  cudaError_t e = launch_ex(k, pl.grid, pl.threads, smem, st, false, p);
  ++g_launches;
  if (e != cudaSuccess) return NPD_ECUDA;
  if (p.want != 0) {
    float* shared_dgate = (p.want & 4) ? static_cast<float*>(a->d_gate) : nullptr;
    e = launch_dim(norm_sums_kernel, dim3(static_cast<unsigned>((a->d + 31) / 32), 2), 1024, 0, st, true, p, pl.grid,
                   a->d_pre_weight, a->d_post_weight, shared_dgate);
    ++g_launches;
  }
  return e == cudaSuccess ? NPD_OK : NPD_ECUDA;
}

}  // extern "C"
