"""ctypes binding of the C-ABI library (include/npd.h).

Argument marshalling only: every step of the computation runs in the library's
CUDA kernels.  PyTorch supplies device memory and streams.  There is no CPU or
PyTorch fallback: if the library is not built the first call raises.
"""

from __future__ import annotations

import contextlib
import ctypes as C
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnpd.so")

NPD_OK = 0
NPD_EINVAL, NPD_ESHAPE, NPD_EALIGN, NPD_ESEQ, NPD_EARCH = -1, -2, -3, -4, -5
NPD_EWORKSPACE, NPD_ECUDA, NPD_ETIMEOUT, NPD_EUNSUPPORTED, NPD_EDATA = -6, -7, -8, -9, -10
NPD_DTYPE_BF16, NPD_DTYPE_F32 = 0, 1
NPD_KD_ACCUMULATE_DW = 1
NPD_KD_COMPOSITE_LOSS = 2
NPD_KD_REVERSE_KL = 4
NPD_KD_SERIALIZE_LAUNCHES = 8
NPD_KD_DEBUG_CHECKS = 16
NPD_SELECT_TEACHER_IFD_LE_1 = 1
NPD_SELECT_SCORE_IFD_TEACHER, NPD_SELECT_SCORE_IFD_STUDENT = 2, 4
NPD_SELECT_LO_EXCLUSIVE, NPD_SELECT_HI_EXCLUSIVE = 8, 16
NPD_NORM_POST = 1
NPD_LINEAR_ACCUMULATE_DW = 1
NPD_ACT_NONE, NPD_ACT_RELU, NPD_ACT_GELU, NPD_ACT_GELU_TANH, NPD_ACT_SILU = range(5)
NPD_CE_ACCUMULATE_DW, NPD_CE_SERIALIZE_LAUNCHES = 1, 2
NPD_GEMM_STORE_F32, NPD_GEMM_ADD_F32, NPD_GEMM_STORE_BF16, NPD_GEMM_ATOMIC_F32 = range(4)

EXPORTS = ("npd_workspace_bytes", "npd_phase_count", "npd_kd_fwd_bwd", "npd_kd_fwd_bwd_host", "npd_segment_stats",
           "npd_select", "npd_last_status", "npd_strerror", "npd_last_launch_count", "npd_gemm_bf16",
           "npd_kd_forward_noalloc", "npd_pack_sequences", "npd_last_copy_bytes",
           "npd_kd_fwd_bwd_host_streams", "npd_perplexity", "npd_selftest_wait_timeout",
           "npd_debug_chunk_schedule", "npd_norm_fwd", "npd_norm_bwd", "npd_norm_workspace_bytes",
           "npd_ce_fwd_bwd", "npd_ce_workspace_bytes", "npd_linear_fwd", "npd_linear_bwd", "npd_linear_workspace_bytes",
           "npd_device_status")
NPD_STATIC_SCRATCH_BYTES = 48 * 1024 * 1024


class NpdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


class npd_kd_args(C.Structure):
    _fields_ = [
        ("size", C.c_size_t),
        ("T", C.c_int32), ("d", C.c_int32), ("V", C.c_int32), ("S", C.c_int32),
        ("hidden", C.c_void_p), ("weight", C.c_void_p), ("teacher", C.c_void_p),
        ("ldh", C.c_int64), ("ldw", C.c_int64), ("ldt", C.c_int64),
        ("teacher_dtype", C.c_int32), ("reserved0", C.c_int32),
        ("cu_seqlens", C.c_void_p), ("loss_mask", C.c_void_p), ("labels", C.c_void_p),
        ("temperature", C.c_float), ("grad_scale", C.c_float),
        ("kl", C.c_void_p), ("nll_student", C.c_void_p), ("nll_teacher", C.c_void_p),
        ("d_hidden", C.c_void_p), ("d_weight", C.c_void_p),
        ("d_weight_dtype", C.c_int32), ("flags", C.c_int32),
        ("grad_chunk_cols", C.c_int32), ("kd_lambda", C.c_float),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
        ("phase_events", C.POINTER(C.c_void_p)), ("n_phase_events", C.c_int32), ("reserved2", C.c_int32),
        ("topk_values", C.c_void_p), ("topk_indices", C.c_void_p), ("topk", C.c_int32), ("reserved3", C.c_int32),
    ]


class npd_norm_args(C.Structure):
    _fields_ = [
        ("size", C.c_size_t), ("T", C.c_int32), ("d", C.c_int32),
        ("stream_dtype", C.c_int32), ("weight_dtype", C.c_int32), ("flags", C.c_int32), ("reserved0", C.c_int32),
        ("eps", C.c_float), ("weight_offset", C.c_float), ("residual_scale", C.c_float), ("branch_scale", C.c_float),
        ("x", C.c_void_p), ("residual", C.c_void_p), ("gate", C.c_void_p),
        ("post_weight", C.c_void_p), ("pre_weight", C.c_void_p), ("h", C.c_void_p), ("y", C.c_void_p),
        ("ldx", C.c_int64), ("ldr", C.c_int64), ("ldg", C.c_int64), ("ldh", C.c_int64), ("ldy", C.c_int64),
        ("dy", C.c_void_p), ("dh", C.c_void_p), ("dx", C.c_void_p), ("dresidual", C.c_void_p), ("d_gate", C.c_void_p),
        ("d_post_weight", C.c_void_p), ("d_pre_weight", C.c_void_p),
        ("lddy", C.c_int64), ("lddh", C.c_int64), ("lddx", C.c_int64), ("lddr", C.c_int64), ("lddg", C.c_int64),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class npd_ce_args(C.Structure):
    _fields_ = [
        ("size", C.c_size_t), ("T", C.c_int32), ("d", C.c_int32), ("V", C.c_int32), ("flags", C.c_int32),
        ("hidden", C.c_void_p), ("weight", C.c_void_p), ("ldh", C.c_int64), ("ldw", C.c_int64),
        ("labels", C.c_void_p), ("loss_mask", C.c_void_p), ("token_weight", C.c_void_p),
        ("temperature", C.c_float), ("grad_scale", C.c_float),
        ("nll", C.c_void_p), ("lse", C.c_void_p), ("d_hidden", C.c_void_p), ("d_weight", C.c_void_p),
        ("ld_dh", C.c_int64), ("ld_dw", C.c_int64),
        ("d_weight_dtype", C.c_int32), ("grad_chunk_cols", C.c_int32),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class npd_linear_args(C.Structure):
    _fields_ = [
        ("size", C.c_size_t), ("M", C.c_int32), ("N", C.c_int32), ("K", C.c_int32), ("activation", C.c_int32),
        ("bias_dtype", C.c_int32), ("y_dtype", C.c_int32), ("dw_dtype", C.c_int32), ("flags", C.c_int32),
        ("x", C.c_void_p), ("weight", C.c_void_p), ("bias", C.c_void_p), ("residual", C.c_void_p), ("y", C.c_void_p),
        ("preact", C.c_void_p),
        ("ldx", C.c_int64), ("ldw", C.c_int64), ("ldr", C.c_int64), ("ldy", C.c_int64), ("ldz", C.c_int64),
        ("dy", C.c_void_p), ("dx", C.c_void_p), ("dw", C.c_void_p), ("dbias", C.c_void_p),
        ("lddy", C.c_int64), ("lddx", C.c_int64), ("lddw", C.c_int64),
        ("status", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


_lib = None


def lib() -> C.CDLL:
    """The loaded library.  Raises if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        from . import build as _build
        if _build.is_stale():          # missing, or built from other sources than the ones present
            _build.build()             # raises if it cannot: never run kernels of other sources
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2605_05940_b200.build` "
                "(there is no CPU or PyTorch fallback)")
        l = C.CDLL(LIB_PATH)
        l.npd_strerror.restype = C.c_char_p
        l.npd_strerror.argtypes = [C.c_int]
        l.npd_workspace_bytes.argtypes = [C.POINTER(npd_kd_args), C.POINTER(C.c_size_t)]
        l.npd_kd_fwd_bwd.argtypes = [C.POINTER(npd_kd_args), C.c_void_p]
        l.npd_phase_count.argtypes = [C.POINTER(npd_kd_args), C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        l.npd_kd_fwd_bwd_host.argtypes = [C.POINTER(npd_kd_args), C.POINTER(npd_kd_args), C.c_void_p]
        l.npd_kd_fwd_bwd_host_streams.argtypes = [C.POINTER(npd_kd_args), C.POINTER(npd_kd_args), C.c_void_p,
                                                  C.c_void_p]
        l.npd_segment_stats.argtypes = [C.c_int32, C.c_int32] + [C.c_void_p] * 13
        l.npd_select.argtypes = ([C.c_int32] + [C.c_void_p] * 5 + [C.c_int32, C.c_float, C.c_float, C.c_int32]
                                 + [C.c_void_p] * 6)
        l.npd_last_status.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int32)]
        l.npd_device_status.argtypes = [C.c_void_p, C.POINTER(C.c_int32)]
        l.npd_last_launch_count.argtypes = []
        l.npd_last_copy_bytes.argtypes = [C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
        l.npd_kd_forward_noalloc.argtypes = [C.POINTER(npd_kd_args), C.c_void_p, C.POINTER(C.c_int32)]
        l.npd_pack_sequences.argtypes = [C.c_int32, C.c_void_p, C.c_void_p, C.c_int32] + [C.c_void_p] * 6
        l.npd_perplexity.argtypes = [C.c_int32] + [C.c_void_p] * 4 + [C.c_int32] + [C.c_void_p] * 3
        l.npd_selftest_wait_timeout.argtypes = [C.c_int64, C.c_void_p, C.c_void_p]
        l.npd_debug_chunk_schedule.argtypes = [C.c_int32] * 6 + [C.c_void_p, C.POINTER(C.c_int32)]
        l.npd_gemm_bf16.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_int32,
                                    C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_int64,
                                    C.c_int32, C.c_int32, C.c_void_p]
        for f in (l.npd_norm_fwd, l.npd_norm_bwd):
            f.argtypes = [C.POINTER(npd_norm_args), C.c_void_p]
        l.npd_norm_workspace_bytes.argtypes = [C.POINTER(npd_norm_args), C.POINTER(C.c_size_t)]
        for f in (l.npd_linear_fwd, l.npd_linear_bwd):
            f.argtypes = [C.POINTER(npd_linear_args), C.c_void_p]
        l.npd_linear_workspace_bytes.argtypes = [C.POINTER(npd_linear_args), C.POINTER(C.c_size_t)]
        l.npd_ce_fwd_bwd.argtypes = [C.POINTER(npd_ce_args), C.c_void_p]
        l.npd_ce_workspace_bytes.argtypes = [C.POINTER(npd_ce_args), C.POINTER(C.c_size_t)]
        _lib = l
    return _lib


def strerror(code: int) -> str:
    return lib().npd_strerror(int(code)).decode()


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(rc: int, where: str):
    if rc != NPD_OK:
        raise NpdError(rc, where)


def make_kd_args(hidden, weight, teacher, *, cu_seqlens=None, loss_mask=None, labels=None,
                 temperature=1.0, grad_scale=1.0, kl=None, nll_student=None, nll_teacher=None,
                 d_hidden=None, d_weight=None, flags=0, grad_chunk_cols=0, kd_lambda=None,
                 topk_values=None, topk_indices=None, workspace=None) -> npd_kd_args:
    """Fill an npd_kd_args from tensors (device tensors, or host tensors for the
    `host` argument of npd_kd_fwd_bwd_host)."""
    a = npd_kd_args()
    a.size = C.sizeof(npd_kd_args)
    a.T, a.d = hidden.shape
    a.V = weight.shape[0]
    a.S = 0 if cu_seqlens is None else cu_seqlens.numel() - 1
    a.hidden, a.weight, a.teacher = _ptr(hidden), _ptr(weight), _ptr(teacher)
    a.ldh, a.ldw = hidden.stride(0), weight.stride(0)
    if teacher is not None:
        a.ldt = teacher.stride(0)
        a.teacher_dtype = NPD_DTYPE_F32 if teacher.dtype == torch.float32 else NPD_DTYPE_BF16
    else:                           # top-k teacher: f32 [T,k] logits and int32 [T,k] indices
        a.ldt = (a.V + 7) // 8 * 8
        a.teacher_dtype = NPD_DTYPE_BF16
    if topk_values is not None:
        a.topk_values, a.topk_indices, a.topk = _ptr(topk_values), _ptr(topk_indices), topk_values.shape[1]
    a.cu_seqlens, a.loss_mask, a.labels = _ptr(cu_seqlens), _ptr(loss_mask), _ptr(labels)
    a.temperature, a.grad_scale = float(temperature), float(grad_scale)
    a.kl, a.nll_student, a.nll_teacher = _ptr(kl), _ptr(nll_student), _ptr(nll_teacher)
    a.d_hidden, a.d_weight = _ptr(d_hidden), _ptr(d_weight)
    a.d_weight_dtype = (NPD_DTYPE_F32 if d_weight is not None and d_weight.dtype == torch.float32
                        else NPD_DTYPE_BF16)
    a.flags, a.grad_chunk_cols = int(flags), int(grad_chunk_cols)
    if kd_lambda is not None:       # composite objective of Eq. 1
        a.flags |= NPD_KD_COMPOSITE_LOSS
        a.kd_lambda = float(kd_lambda)
    if workspace is not None:
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    return a


def npd_workspace_bytes(args: npd_kd_args) -> int:
    out = C.c_size_t(0)
    _check(lib().npd_workspace_bytes(C.byref(args), C.byref(out)), "npd_workspace_bytes")
    return out.value


def npd_phase_count(args: npd_kd_args):
    """(launch groups, vocabulary chunks) of a call with these arguments."""
    g, c = C.c_int32(0), C.c_int32(0)
    _check(lib().npd_phase_count(C.byref(args), C.byref(g), C.byref(c)), "npd_phase_count")
    return g.value, c.value


def npd_kd_fwd_bwd(args: npd_kd_args, stream=None) -> None:
    _check(lib().npd_kd_fwd_bwd(C.byref(args), _stream(stream)), "npd_kd_fwd_bwd")


def npd_kd_fwd_bwd_host(host: npd_kd_args, dev: npd_kd_args, stream=None) -> None:
    _check(lib().npd_kd_fwd_bwd_host(C.byref(host), C.byref(dev), _stream(stream)), "npd_kd_fwd_bwd_host")


def npd_kd_fwd_bwd_host_streams(host: npd_kd_args, dev: npd_kd_args, copy_stream, stream=None) -> None:
    _check(lib().npd_kd_fwd_bwd_host_streams(C.byref(host), C.byref(dev), _stream(copy_stream), _stream(stream)),
           "npd_kd_fwd_bwd_host_streams")


def npd_kd_forward_noalloc(args: npd_kd_args, stream=None, want_status: bool = False):
    """Forward pass on the library's built-in scratch array (no workspace, no allocation).
    For callers that cannot allocate device memory; see include/npd.h for the limits.
    With want_status the call synchronises the stream and returns the device status."""
    st = C.c_int32(0)
    _check(lib().npd_kd_forward_noalloc(C.byref(args), _stream(stream), C.byref(st) if want_status else None),
           "npd_kd_forward_noalloc")
    return st.value if want_status else None


def npd_last_status(workspace: torch.Tensor, stream=None) -> int:
    out = C.c_int32(0)
    _check(lib().npd_last_status(workspace.data_ptr(), _stream(stream), C.byref(out)), "npd_last_status")
    return out.value


def npd_device_status(device=None, stream=None) -> int:
    """Waits for `stream` (default: the current one) and returns NPD_ETIMEOUT if a bounded wait of any kernel of the
    library on this GPU (default: the current one) has run out since the last time this was asked, else NPD_OK.  For the
    calls that keep no status word for their caller: npd_gemm_bf16, npd_linear_fwd and npd_linear_bwd, npd_cross_entropy."""
    out = C.c_int32(0)
    index = device if isinstance(device, int) else None if device is None else torch.device(device).index
    if index is None:
        index = torch.cuda.current_device()
    with _scope(index, stream):
        _check(lib().npd_device_status(_current(index), C.byref(out)), "npd_device_status")
    return out.value


def npd_last_launch_count() -> int:
    return lib().npd_last_launch_count()


def npd_last_copy_bytes():
    """(host-to-device, device-to-host) bytes of the last npd_kd_fwd_bwd_host call on this thread."""
    a, b = C.c_int64(0), C.c_int64(0)
    _check(lib().npd_last_copy_bytes(C.byref(a), C.byref(b)), "npd_last_copy_bytes")
    return a.value, b.value


def npd_segment_stats(cu_seqlens, loss_mask, labels, kl, nll_student, nll_teacher, *,
                      kl_sum=None, nll_s_sum=None, nll_t_sum=None, count=None, seg_id=None,
                      status=None, stream=None):
    """Per-segment sums and counts.  Allocates the outputs that are not given and
    returns (kl_sum, nll_s_sum, nll_t_sum, count, seg_id)."""
    S = cu_seqlens.numel() - 1
    ref = next(t for t in (kl, nll_student, nll_teacher, loss_mask, labels, cu_seqlens) if t is not None)
    T = ref.numel() if ref is not cu_seqlens else int(cu_seqlens[-1].item())
    dev = cu_seqlens.device
    f = lambda src, out: (torch.empty(S, dtype=torch.float32, device=dev) if out is None and src is not None else out)
    kl_sum, nll_s_sum, nll_t_sum = f(kl, kl_sum), f(nll_student, nll_s_sum), f(nll_teacher, nll_t_sum)
    if count is None:
        count = torch.empty(S, dtype=torch.int32, device=dev)
    if seg_id is None:
        seg_id = torch.empty(T, dtype=torch.int32, device=dev)
    _check(lib().npd_segment_stats(T, S, _ptr(cu_seqlens), _ptr(loss_mask), _ptr(labels), _ptr(kl),
                                   _ptr(nll_student), _ptr(nll_teacher), _ptr(kl_sum), _ptr(nll_s_sum),
                                   _ptr(nll_t_sum), _ptr(count), _ptr(seg_id), _ptr(status),
                                   _stream(stream)), "npd_segment_stats")
    return kl_sum, nll_s_sum, nll_t_sum, count, seg_id


def npd_select(cond_seg, uncond_seg, nll_s_sum, nll_t_sum, count, lo: float, hi: float, flags: int = 0,
               stream=None):
    """Delta-IFD scores and keep mask.  Returns (ifd_teacher, ifd_student, delta, keep, n_keep)."""
    N, S, dev = cond_seg.numel(), count.numel(), cond_seg.device
    ifd_t = torch.empty(N, dtype=torch.float32, device=dev)
    ifd_s = torch.empty(N, dtype=torch.float32, device=dev)
    delta = torch.empty(N, dtype=torch.float32, device=dev)
    keep = torch.empty(N, dtype=torch.uint8, device=dev)
    n_keep = torch.empty(1, dtype=torch.int32, device=dev)
    _check(lib().npd_select(N, _ptr(cond_seg), _ptr(uncond_seg), _ptr(nll_s_sum), _ptr(nll_t_sum),
                            _ptr(count), S, float(lo), float(hi), int(flags), _ptr(ifd_t), _ptr(ifd_s),
                            _ptr(delta), _ptr(keep), _ptr(n_keep), _stream(stream)), "npd_select")
    return ifd_t, ifd_s, delta, keep, n_keep


def npd_perplexity(seg, nll_s_sum, nll_t_sum, count, stream=None):
    """Per-sample perplexities exp(nll_sum / count) of the segments `seg`.  Returns
    (ppl_student, ppl_teacher); an output is None when its sums are None."""
    N, S, dev = seg.numel(), count.numel(), seg.device
    ps = torch.empty(N, dtype=torch.float32, device=dev) if nll_s_sum is not None else None
    pt = torch.empty(N, dtype=torch.float32, device=dev) if nll_t_sum is not None else None
    _check(lib().npd_perplexity(N, _ptr(seg), _ptr(nll_s_sum), _ptr(nll_t_sum), _ptr(count), S, _ptr(ps),
                                _ptr(pt), _stream(stream)), "npd_perplexity")
    return ps, pt


def npd_selftest_wait_timeout(limit_cycles: int, device="cuda", stream=None):
    """Runs the time-out path of the bounded device waits on purpose (see include/npd.h).
    Returns the int32[3] device tensor {status, every wait gave up, cycles waited}."""
    out = torch.empty(3, dtype=torch.int32, device=device)
    _check(lib().npd_selftest_wait_timeout(int(limit_cycles), _ptr(out), _stream(stream)),
           "npd_selftest_wait_timeout")
    return out


def npd_debug_chunk_schedule(row_blocks: int, d: int, chunk_cols: int, pairs: int, pair: int):
    """Host only: the (problem, row, column, k-step begin, k-step end) units of one CTA pair in the
    launch of a chunk's two backward contractions, as an int32 array [n, 5]."""
    import numpy as np
    n = C.c_int32(0)
    cap = 64
    while True:
        units = np.empty((cap, 5), np.int32)
        _check(lib().npd_debug_chunk_schedule(row_blocks, d, chunk_cols, pairs, pair, cap, units.ctypes.data,
                                              C.byref(n)), "npd_debug_chunk_schedule")
        if n.value <= cap:
            return units[: n.value].copy()
        cap = n.value


def npd_pack_sequences(lengths, keep, capacity: int):
    """First-fit-decreasing packing of the kept samples into rows of `capacity` tokens (host only).
    lengths: int32 array-like, keep: uint8 array-like or None.  Returns numpy arrays
    (order, row_of, cu_seqlens, row_ptr)."""
    import numpy as np
    lengths = np.ascontiguousarray(lengths, dtype=np.int32)
    N = lengths.size
    k = None if keep is None else np.ascontiguousarray(keep, dtype=np.uint8)
    order, row_of = np.empty(N, np.int32), np.empty(N, np.int32)
    cu, ptr = np.empty(N + 1, np.int32), np.empty(N + 1, np.int32)
    placed, rows = C.c_int32(0), C.c_int32(0)
    _check(lib().npd_pack_sequences(N, lengths.ctypes.data, None if k is None else k.ctypes.data, int(capacity),
                                    order.ctypes.data, row_of.ctypes.data, cu.ctypes.data, ptr.ctypes.data,
                                    C.addressof(placed), C.addressof(rows)), "npd_pack_sequences")
    return order[:placed.value], row_of[:placed.value], cu[:placed.value + 1], ptr[:rows.value + 1]


def npd_gemm_bf16(A, B, out, *, a_mn_major=False, b_mn_major=False, out_mode=NPD_GEMM_STORE_F32,
                  k_splits=1, stream=None):
    """out[M,N] (+)= sum_k A[m,k] B[n,k].  A is [M,K] (K-major) or [K,M] (MN-major); same for B."""
    M, N = out.shape
    K = A.shape[0] if a_mn_major else A.shape[1]
    _check(lib().npd_gemm_bf16(M, N, K, _ptr(A), A.stride(0), int(a_mn_major), _ptr(B), B.stride(0),
                               int(b_mn_major), _ptr(out), out.stride(0), int(out_mode), int(k_splits),
                               _stream(stream)), "npd_gemm_bf16")
    return out


# ----------------------------------------------------------------------------------------------
# Checks and allocations shared by the calls below, which take tensors and return their results.
# Written for little host time: a call on a small problem is bound by what Python does around it.
# ----------------------------------------------------------------------------------------------
_DT = {torch.bfloat16: NPD_DTYPE_BF16, torch.float32: NPD_DTYPE_F32}
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None


def _device_of(t, where):
    """Index of the GPU that holds t; a missing tensor or one elsewhere is refused."""
    if t is None or not t.is_cuda:
        raise NpdError(NPD_EINVAL, where)
    return t.get_device()


def _matrix(t, where, dev, shape, dtype):
    """Checks an operand of this shape and type on GPU `dev` and returns its row stride."""
    if t.dtype is not dtype or t.get_device() != dev:
        raise NpdError(NPD_EINVAL, where)
    if t.shape != shape:
        raise NpdError(NPD_ESHAPE, where)
    rows, cols = shape
    s = t.stride()
    if cols > 1 and s[1] != 1:
        raise NpdError(NPD_ESHAPE, where)
    return s[0] if rows > 1 else (cols + 7) // 8 * 8     # the stride of a single row is never used


def _vector(t, where, dev, n, dtype):
    """Checks a contiguous vector of n elements on GPU `dev` and returns its address."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != dev:
        raise NpdError(NPD_EINVAL, where)
    if t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise NpdError(NPD_ESHAPE, where)
    return t.data_ptr()


def _touch(a, b):
    """Whether two tensors share a byte.  Column windows of one wider buffer may lie between each other's rows."""
    if a is None or b is None or a.get_device() != b.get_device():
        return False
    span = lambda t: (1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride()))) * t.element_size()
    a0, b0 = a.data_ptr(), b.data_ptr()
    if a0 + span(a) <= b0 or b0 + span(b) <= a0:
        return False
    if a.dim() != 2 or b.dim() != 2:
        return True
    pitch, wa, wb = (v * t.element_size() for t, v in ((a, a.stride(0)), (a, a.shape[1]), (b, b.shape[1])))
    if pitch != b.stride(0) * b.element_size() or max(wa, wb) > pitch:
        return True
    delta = (b0 - a0) % pitch
    return delta < wa or pitch - delta < wb


def _new(shape, dtype, device):
    """An uninitialised matrix whose rows start on 16-byte boundaries."""
    cols = shape[1]
    if cols % 8 == 0:
        return torch.empty(shape, dtype=dtype, device=device)
    return torch.empty_strided(shape, ((cols + 7) // 8 * 8, 1), dtype=dtype, device=device)


def _like(t, shape, dtype):
    """_new(...) on t's GPU; quicker where t itself has that shape and type and is dense."""
    if t is not None and t.dtype is dtype and shape[1] % 8 == 0 and t.is_contiguous():
        return torch.empty_like(t)
    return None if t is None else _new(shape, dtype, t.device)


_no_scope = contextlib.nullcontext()


def _scope(dev, stream):
    """The device of the operands current and, if a stream is given, torch's allocations on it: what a
    call allocates belongs to the stream that the call runs on."""
    if stream is None:
        return _no_scope if dev == torch.cuda.current_device() else torch.cuda.device(dev)
    if not hasattr(stream, "cuda_stream"):
        # handle 0 is the default stream; ExternalStream(0) would be another one, out of torch's pool
        stream = torch.cuda.ExternalStream(int(stream), device=dev) if int(stream) else torch.cuda.default_stream(dev)
    if stream.device.index != dev:
        raise NpdError(NPD_EINVAL, "stream of another device")
    return torch.cuda.stream(stream)


def _current(dev):
    """Handle of torch's current stream on GPU `dev`."""
    return _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream(dev).cuda_stream


def _workspace(nbytes, device):
    """`nbytes` of device memory, and the address of the first 1024-byte boundary in it."""
    t = torch.empty(nbytes + 1024, dtype=torch.uint8, device=device)
    return t, (t.data_ptr() + 1023) & ~1023


def _given_workspace(t, where, dev):
    """Address and size in bytes of a caller's workspace: dense memory on GPU `dev`.  The library checks its size and
    alignment, but takes the address on trust."""
    if t.get_device() != dev or not t.is_contiguous():
        raise NpdError(NPD_EWORKSPACE, where)
    return t.data_ptr(), t.numel() * t.element_size()


def _norm_args(where, dev, shape, x, gate, post_weight, pre_weight, post_norm, eps, weight_offset, residual_scale,
               branch_scale, stream_dtype):
    T, d = shape
    w = post_weight if post_weight is not None else pre_weight
    if stream_dtype not in _DT or (w is not None and w.dtype not in _DT):
        raise NpdError(NPD_EINVAL, where)
    a = npd_norm_args(C.sizeof(npd_norm_args), T, d, _DT[stream_dtype], 0 if w is None else _DT[w.dtype],
                      NPD_NORM_POST if post_norm else 0, 0, eps, weight_offset, residual_scale, branch_scale)
    if w is not None:
        a.post_weight = _vector(post_weight, where, dev, d, w.dtype)
        a.pre_weight = _vector(pre_weight, where, dev, d, w.dtype)
    if x is not None:
        a.ldx, a.x = _matrix(x, where, dev, shape, torch.bfloat16), x.data_ptr()
    if gate is not None:
        if gate.dim() == 1:
            a.gate = _vector(gate, where, dev, d, torch.bfloat16)
        else:
            a.ldg, a.gate = _matrix(gate, where, dev, shape, torch.bfloat16), gate.data_ptr()
            if a.ldg < d:          # rows expanded from one: a shared gate is passed as a vector
                raise NpdError(NPD_ESHAPE, where)
    return a


def npd_norm_fwd(x, residual=None, *, gate=None, post_weight=None, pre_weight=None, post_norm=False, eps=1e-6,
                 weight_offset=0.0, residual_scale=1.0, branch_scale=1.0, want_h=True, want_y=True, h=None, y=None,
                 stream=None):
    """h = residual_scale * residual + branch_scale * gate * (norm of x, or x) and y = norm of h (see
    npd_norm_args in include/npd.h).  x bf16 [T, d] or None, residual bf16 or f32 [T, d] or None, gate bf16
    [d] (shared) or [T, d]; gains [d].  Results go to h and y, or to new tensors (want_h / want_y);
    returns (h, y).  Allocations and kernels use `stream` (default: the current one)."""
    where = "npd_norm_fwd"
    first = x if x is not None else residual
    dev = _device_of(first, where)
    shape = first.shape
    if len(shape) != 2:
        raise NpdError(NPD_ESHAPE, where)
    sd = residual.dtype if residual is not None else (h.dtype if h is not None else torch.bfloat16)
    with _scope(dev, stream):
        a = _norm_args(where, dev, shape, x, gate, post_weight, pre_weight, post_norm, eps, weight_offset,
                       residual_scale, branch_scale, sd)
        if residual is not None:
            a.ldr, a.residual = _matrix(residual, where, dev, shape, sd), residual.data_ptr()
        if h is None and want_h:
            h = _like(residual if residual is not None else first, shape, sd)
        if y is None and want_y:
            y = _like(first, shape, torch.bfloat16)
        if h is not None:
            a.ldh, a.h = _matrix(h, where, dev, shape, sd), h.data_ptr()
        if y is not None:
            a.ldy, a.y = _matrix(y, where, dev, shape, torch.bfloat16), y.data_ptr()
        _check(lib().npd_norm_fwd(a, _current(dev)), where)
    return h, y


def npd_norm_bwd(dy, h, x=None, *, dh=None, gate=None, post_weight=None, pre_weight=None, post_norm=False, eps=1e-6,
                 weight_offset=0.0, residual_scale=1.0, branch_scale=1.0, want_dresidual=True, want_dweights=True,
                 dx=None, dresidual=None, d_post_weight=None, d_pre_weight=None, d_gate=None, workspace=None, stream=None):
    """Gradients of npd_norm_fwd.  dy is the gradient at y (or None), h the forward's h, dh the gradient that
    arrives at h from elsewhere (or None); the rest as in the forward.  Returns (dx, dresidual,
    d_post_weight, d_pre_weight, d_gate) in the tensors given or in new ones, None for what has no counterpart in
    the call; the gradients of the gains and of a shared gate are f32 [d] sums over the tokens."""
    where = "npd_norm_bwd"
    first = dy if dy is not None else dh
    dev = _device_of(first, where)
    shape, device = first.shape, first.device
    if len(shape) != 2:
        raise NpdError(NPD_ESHAPE, where)
    T, d = shape
    sd = next((t.dtype for t in (h, dh, dresidual) if t is not None), torch.bfloat16)
    bf16 = torch.bfloat16
    with _scope(dev, stream):
        a = _norm_args(where, dev, shape, x, gate, post_weight, pre_weight, post_norm, eps, weight_offset,
                       residual_scale, branch_scale, sd)
        if dy is not None:
            a.lddy, a.dy = _matrix(dy, where, dev, shape, bf16), dy.data_ptr()
        if h is not None:
            a.ldh, a.h = _matrix(h, where, dev, shape, sd), h.data_ptr()
        if dh is not None:
            a.lddh, a.dh = _matrix(dh, where, dev, shape, sd), dh.data_ptr()
        if dx is None and x is not None:
            dx = _like(x, shape, bf16)
        if dresidual is None and want_dresidual:
            dresidual = _like(dh if dh is not None else first, shape, sd)
        if dx is not None:
            a.lddx, a.dx = _matrix(dx, where, dev, shape, bf16), dx.data_ptr()
        if dresidual is not None:
            a.lddr, a.dresidual = _matrix(dresidual, where, dev, shape, sd), dresidual.data_ptr()
        d_post, d_pre = d_post_weight, d_pre_weight
        if d_post is None and want_dweights and post_norm and post_weight is not None:
            d_post = torch.empty(d, dtype=torch.float32, device=device)
        if d_pre is None and want_dweights and pre_weight is not None and dy is not None:
            d_pre = torch.empty(d, dtype=torch.float32, device=device)
        a.d_post_weight = _vector(d_post, where, dev, d, torch.float32)
        a.d_pre_weight = _vector(d_pre, where, dev, d, torch.float32)
        shared = gate is not None and gate.dim() == 1
        if shared:
            if d_gate is None:
                d_gate = torch.empty(d, dtype=torch.float32, device=device)
            a.d_gate = _vector(d_gate, where, dev, d, torch.float32)
        elif gate is not None:
            if d_gate is None:
                d_gate = _new(shape, bf16, device)
            a.lddg, a.d_gate = _matrix(d_gate, where, dev, shape, bf16), d_gate.data_ptr()
        elif d_gate is not None:
            raise NpdError(NPD_EINVAL, where)
        if d_post is not None or d_pre is not None or shared:
            if workspace is None:
                n = C.c_size_t(0)
                _check(lib().npd_norm_workspace_bytes(a, n), where)
                workspace, a.workspace = _workspace(n.value, device)
                a.workspace_bytes = n.value
            else:
                a.workspace, a.workspace_bytes = _given_workspace(workspace, where, dev)
        _check(lib().npd_norm_bwd(a, _current(dev)), where)
    return dx, dresidual, d_post, d_pre, d_gate


def npd_linear_fwd(x, weight, *, bias=None, activation=NPD_ACT_NONE, residual=None, want_preact=False,
                   y_dtype=torch.bfloat16, y=None, preact=None, status=None, stream=None):
    """y = act(x weight^T + bias) + residual (see npd_linear_args in include/npd.h).  x bf16 [M, K], weight bf16
    [N, K], bias bf16 or f32 [N], residual of y's type [M, N].  Results go to y and preact or to new tensors
    (want_preact: the bf16 pre-activation that the backward needs); returns (y, preact).  A wait that ran out on the
    device shows in `status`, int32[1], and in npd_device_status."""
    where = "npd_linear_fwd"
    dev = _device_of(x, where)
    if x.dim() != 2 or weight.dim() != 2:
        raise NpdError(NPD_ESHAPE, where)
    (M, K), N, bf16 = x.shape, weight.shape[0], torch.bfloat16
    if y is not None:
        y_dtype = y.dtype
    elif residual is not None:
        y_dtype = residual.dtype
    if y_dtype not in _DT or (bias is not None and bias.dtype not in _DT):
        raise NpdError(NPD_EINVAL, where)
    with _scope(dev, stream):
        a = npd_linear_args(C.sizeof(npd_linear_args), M, N, K, activation, 0 if bias is None else _DT[bias.dtype],
                            _DT[y_dtype])
        a.ldx, a.x = _matrix(x, where, dev, (M, K), bf16), x.data_ptr()
        a.ldw, a.weight = _matrix(weight, where, dev, (N, K), bf16), weight.data_ptr()
        if bias is not None:
            a.bias = _vector(bias, where, dev, N, bias.dtype)
        if residual is not None:
            a.ldr, a.residual = _matrix(residual, where, dev, (M, N), y_dtype), residual.data_ptr()
        if y is None:
            y = _new((M, N), y_dtype, x.device)
        a.ldy, a.y = _matrix(y, where, dev, (M, N), y_dtype), y.data_ptr()
        if preact is None and want_preact:
            preact = _new((M, N), bf16, x.device)
        if preact is not None:
            a.ldz, a.preact = _matrix(preact, where, dev, (M, N), bf16), preact.data_ptr()
        if status is not None:
            a.status = _vector(status, where, dev, 1, torch.int32)
        _check(lib().npd_linear_fwd(a, _current(dev)), where)
    return y, preact


def npd_linear_bwd(dy, x, weight, *, preact=None, activation=NPD_ACT_NONE, want_dx=True, want_dw=True, want_dbias=False,
                   dw_dtype=torch.bfloat16, dx=None, dw=None, accumulate_dw=False, workspace=None, stream=None):
    """Gradients of npd_linear_fwd from dy bf16 [M, N]: (dx bf16 [M, K], dw [N, K], dbias f32 [N]), None for what
    is not wanted.  preact is the forward's (not needed without an activation), x only for dw.  An f32 dw with
    accumulate_dw is added to (a new one starts at zero).  The gradient of the residual is dy itself.  A wait that ran
    out on the device shows in npd_device_status, and in a workspace of the caller's (npd_last_status)."""
    where = "npd_linear_bwd"
    dev = _device_of(dy, where)
    if dy.dim() != 2 or weight is None or weight.dim() != 2:
        raise NpdError(NPD_ESHAPE, where)
    (M, N), K, device, bf16 = dy.shape, weight.shape[1], dy.device, torch.bfloat16
    if dw is not None:
        dw_dtype = dw.dtype
    if dw_dtype not in _DT:
        raise NpdError(NPD_EINVAL, where)
    with _scope(dev, stream):
        a = npd_linear_args(C.sizeof(npd_linear_args), M, N, K, activation, 0, 0, _DT[dw_dtype],
                            NPD_LINEAR_ACCUMULATE_DW if accumulate_dw else 0)
        a.lddy, a.dy = _matrix(dy, where, dev, (M, N), bf16), dy.data_ptr()
        a.ldw, a.weight = _matrix(weight, where, dev, (N, K), bf16), weight.data_ptr()
        if x is not None:
            a.ldx, a.x = _matrix(x, where, dev, (M, K), bf16), x.data_ptr()
        if preact is not None:
            a.ldz, a.preact = _matrix(preact, where, dev, (M, N), bf16), preact.data_ptr()
        if dx is None and want_dx:
            dx = _new((M, K), bf16, device)
        if dx is not None:
            a.lddx, a.dx = _matrix(dx, where, dev, (M, K), bf16), dx.data_ptr()
        if dw is None and want_dw:
            dw = _new((N, K), dw_dtype, device)
            if accumulate_dw:
                dw.zero_()
        if dw is not None:
            a.lddw, a.dw = _matrix(dw, where, dev, (N, K), dw_dtype), dw.data_ptr()
        dbias = torch.empty(N, dtype=torch.float32, device=device) if want_dbias else None
        a.dbias = _ptr(dbias)
        if workspace is None:
            n = C.c_size_t(0)
            _check(lib().npd_linear_workspace_bytes(a, n), where)
            workspace, a.workspace = _workspace(n.value, device)
            a.workspace_bytes = n.value
        else:
            a.workspace, a.workspace_bytes = _given_workspace(workspace, where, dev)
        _check(lib().npd_linear_bwd(a, _current(dev)), where)
    return dx, dw, dbias


class NormJoin:
    """What stands between a student's last block and its LM head: h = residual_scale * residual +
    branch_scale * gate * (norm of x, or x), hidden states = norm of h (npd_norm_fwd / npd_norm_bwd), with its
    buffers.  Given to KDStep or CEStep as `norm`, every run of the step first writes the step's hidden states and
    afterwards turns their gradient into those of x, residual, gate and gains: dx, dresidual, d_post_weight,
    d_pre_weight, d_gate.  For a step without d_hidden (scoring, a head trained alone) the join is made with
    grads=False; otherwise the step refuses it.  The backward reads x, gate and gains again, so the step's hidden
    states and d_hidden lie apart from them (hidden may be x's memory with grads=False).  The buffers belong to one
    run at a time.  Arguments as for npd_norm_fwd."""

    def __init__(self, x, residual=None, *, grads=True, **how):
        self.x, self.residual, self.how, self.grads = x, residual, how, grads
        first = x if x is not None else residual
        dev = _device_of(first, "NormJoin")
        shape, device = first.shape, first.device
        if len(shape) != 2:
            raise NpdError(NPD_ESHAPE, "NormJoin")
        with _scope(dev, None):
            sd = residual.dtype if residual is not None else torch.bfloat16
            self.h = _new(shape, sd, device)
            self.dx = self.dresidual = self.d_post_weight = self.d_pre_weight = self.d_gate = None
            if not grads:
                return
            d, gate = shape[1], how.get("gate")
            f32 = lambda: torch.empty(d, dtype=torch.float32, device=device)
            if x is not None:
                self.dx = _new(shape, torch.bfloat16, device)
            if residual is not None:
                self.dresidual = _new(shape, sd, device)
            if how.get("post_norm") and how.get("post_weight") is not None:
                self.d_post_weight = f32()
            if how.get("pre_weight") is not None:
                self.d_pre_weight = f32()
            if gate is not None:
                self.d_gate = f32() if gate.dim() == 1 else _new(shape, torch.bfloat16, device)
            a = npd_norm_args(C.sizeof(npd_norm_args), shape[0], d, _DT[sd])
            n = C.c_size_t(0)
            _check(lib().npd_norm_workspace_bytes(a, n), "npd_norm_workspace_bytes")
            self._workspace = torch.empty(n.value, dtype=torch.uint8, device=device)

    def attach(self, hidden, d_hidden):
        """What a step checks when it is made.  Gradients that no run would write are refused (their buffers would pass
        for results), and so are steps that write over what the backward reads after them."""
        if not self.grads:
            return
        if d_hidden is None:
            raise NpdError(NPD_EINVAL, "NormJoin: gradients of a step without d_hidden")
        for t in (self.x, *(self.how.get(k) for k in ("gate", "post_weight", "pre_weight"))):
            if _touch(hidden, t) or _touch(d_hidden, t):
                raise NpdError(NPD_EINVAL, "NormJoin: the step writes over an operand of the join")

    def forward(self, hidden, stream=None):
        npd_norm_fwd(self.x, self.residual, h=self.h, y=hidden, stream=stream, **self.how)

    def backward(self, d_hidden, stream=None):
        npd_norm_bwd(d_hidden, self.h, self.x, dx=self.dx, dresidual=self.dresidual, want_dresidual=False,
                     d_post_weight=self.d_post_weight, d_pre_weight=self.d_pre_weight, d_gate=self.d_gate,
                     workspace=self._workspace, stream=stream, **self.how)


class CEStep:
    """Cross-entropy of the LM head for one set of tensors: checks them, holds the results (nll, lse,
    d_hidden, d_weight) and the workspace, and runs the step on them; see npd_ce_args in include/npd.h.

    hidden bf16 [T, d], weight bf16 [V, d], labels int32 [T], loss_mask uint8 or bool [T], token_weight f32 [T].
    norm: a NormJoin that writes `hidden` before, and takes d_hidden back after the step.
    d_hidden / d_weight: True for a new tensor, None for none, or a tensor to write to (an f32 d_weight with
    accumulate_dw is added to by every run; a new one starts at zero).  The tensors are allocated on `stream` (default: the current one)."""

    def __init__(self, hidden, weight, labels, *, loss_mask=None, token_weight=None, temperature=1.0, grad_scale=1.0,
                 d_hidden=True, d_weight=True, dw_dtype=torch.bfloat16, accumulate_dw=False, want_lse=True,
                 grad_chunk_cols=0, flags=0, workspace=None, norm=None, stream=None):
        where = "npd_ce_fwd_bwd"
        self.norm = norm
        dev = self._dev = _device_of(hidden, where)
        if hidden.dim() != 2 or weight.dim() != 2:
            raise NpdError(NPD_ESHAPE, where)
        shape, device, bf16 = hidden.shape, hidden.device, torch.bfloat16
        T, d = shape
        V = weight.shape[0]
        a = self.args = npd_ce_args(C.sizeof(npd_ce_args), T, d, V, flags | (NPD_CE_ACCUMULATE_DW if accumulate_dw else 0))
        # what the step reads is kept alive as long as the step is
        self._inputs = (hidden, weight, labels, loss_mask, token_weight)
        with _scope(dev, stream):
            a.ldh, a.hidden = _matrix(hidden, where, dev, shape, bf16), hidden.data_ptr()
            a.ldw, a.weight = _matrix(weight, where, dev, (V, d), bf16), weight.data_ptr()
            a.labels = _vector(labels, where, dev, T, torch.int32)
            if loss_mask is not None:
                a.loss_mask = _vector(loss_mask, where, dev, T, torch.bool if loss_mask.dtype is torch.bool else torch.uint8)
            a.token_weight = _vector(token_weight, where, dev, T, torch.float32)
            a.temperature, a.grad_scale, a.grad_chunk_cols = temperature, grad_scale, grad_chunk_cols
            self.nll = torch.empty(T, dtype=torch.float32, device=device)
            self.lse = torch.empty(T, dtype=torch.float32, device=device) if want_lse else None
            a.nll, a.lse = self.nll.data_ptr(), _ptr(self.lse)
            if d_hidden is True:
                d_hidden = _like(hidden, shape, bf16)
            if d_weight is True:
                d_weight = _new((V, d), dw_dtype, device)
                if accumulate_dw:
                    d_weight.zero_()
            self.d_hidden, self.d_weight = d_hidden, d_weight
            if norm is not None:
                norm.attach(hidden, d_hidden)
            if d_hidden is not None:
                a.ld_dh, a.d_hidden = _matrix(d_hidden, where, dev, shape, bf16), d_hidden.data_ptr()
            if d_weight is not None:
                if d_weight.dtype not in _DT:
                    raise NpdError(NPD_EINVAL, where)
                a.ld_dw, a.d_weight = _matrix(d_weight, where, dev, (V, d), d_weight.dtype), d_weight.data_ptr()
                a.d_weight_dtype = _DT[d_weight.dtype]
            if workspace is None:
                n = C.c_size_t(0)
                _check(lib().npd_ce_workspace_bytes(a, n), where)
                self._workspace, a.workspace = _workspace(n.value, device)
                a.workspace_bytes = n.value
            else:
                self._workspace = workspace
                a.workspace, a.workspace_bytes = _given_workspace(workspace, where, dev)

    def run(self, stream=None):
        """Enqueues the step on `stream` (default: the current one of the tensors' GPU)."""
        if self.norm is not None:
            self.norm.forward(self._inputs[0], stream)
        with _scope(self._dev, stream):
            _check(lib().npd_ce_fwd_bwd(self.args, _current(self._dev)), "npd_ce_fwd_bwd")
        if self.norm is not None and self.norm.grads:
            self.norm.backward(self.d_hidden, stream)

    def status(self, stream=None) -> int:
        """Waits for `stream` and returns the status that the step's kernels left in the workspace."""
        out = C.c_int32(0)
        with _scope(self._dev, stream):
            _check(lib().npd_last_status(self.args.workspace, _current(self._dev), C.byref(out)), "npd_last_status")
        return out.value


def npd_cross_entropy(hidden, weight, labels, *, grads=True, stream=None, **kw):
    """One cross-entropy step with new results: (nll, lse, d_hidden, d_weight), the gradients None without
    `grads`.  Further arguments as for CEStep, which a loop over fixed buffers uses instead.  A wait that ran out on
    the device shows in npd_device_status."""
    if not grads:
        kw["d_hidden"] = kw["d_weight"] = None
    s = CEStep(hidden, weight, labels, stream=stream, **kw)
    s.run(stream)
    return s.nll, s.lse, s.d_hidden, s.d_weight


class KDStep:
    """Holds the output and workspace tensors of one problem shape and runs the
    fused step on them; a convenience over the raw calls."""

    def __init__(self, batch, *, grads=True, dw_dtype=torch.bfloat16, grad_chunk_cols=0, grad_scale=None,
                 kd_lambda=None, topk_values=None, topk_indices=None, flags=0, norm=None):
        self.norm = norm   # a NormJoin that writes batch.hidden before, and takes d_hidden back after the step
        # the tensors whose addresses the step keeps, whatever the batch holds later
        self._inputs = (batch.hidden, batch.weight, batch.teacher if topk_values is None else None, batch.cu_seqlens,
                        batch.loss_mask, batch.labels)
        dev = batch.hidden.device
        T, d, V = batch.T, batch.d, batch.V
        f32 = dict(dtype=torch.float32, device=dev)
        self.batch = batch
        self.kl = torch.empty(T, **f32)
        self.nll_student = torch.empty(T, **f32)
        self.nll_teacher = torch.empty(T, **f32) if topk_values is None else None
        self.topk_values, self.topk_indices = topk_values, topk_indices
        # the gradients use the row strides of the tensors they belong to (ldh, ldw)
        self.d_hidden = (torch.empty_strided((T, d), (batch.hidden.stride(0), 1), dtype=torch.bfloat16,
                                             device=dev) if grads else None)
        self.d_weight = (torch.empty_strided((V, d), (batch.weight.stride(0), 1), dtype=dw_dtype,
                                             device=dev) if grads else None)
        if norm is not None:
            norm.attach(batch.hidden, self.d_hidden)
        self.grad_scale = (1.0 / max(batch.n_loss, 1)) if grad_scale is None else grad_scale
        self._kw = dict(cu_seqlens=batch.cu_seqlens, loss_mask=batch.loss_mask, labels=batch.labels,
                        temperature=batch.tau, grad_scale=self.grad_scale, kl=self.kl,
                        nll_student=self.nll_student, nll_teacher=self.nll_teacher,
                        d_hidden=self.d_hidden, d_weight=self.d_weight, grad_chunk_cols=grad_chunk_cols,
                        kd_lambda=kd_lambda, topk_values=topk_values, topk_indices=topk_indices,
                        flags=flags)
        teacher = batch.teacher if topk_values is None else None
        probe = make_kd_args(batch.hidden, batch.weight, teacher, **self._kw)
        nbytes = npd_workspace_bytes(probe)
        self.workspace = torch.empty(nbytes + 1024, dtype=torch.uint8, device=dev)
        off = (-self.workspace.data_ptr()) % 1024
        self._ws_view = self.workspace[off: off + nbytes]
        self.args = make_kd_args(batch.hidden, batch.weight, teacher, workspace=self._ws_view,
                                 **self._kw)

    def run(self, stream=None):
        self._run(self.args, stream)

    def _run(self, args, stream):
        if self.norm is not None:
            self.norm.forward(self._inputs[0], stream)
        npd_kd_fwd_bwd(args, stream)
        if self.norm is not None and self.norm.grads:
            self.norm.backward(self.d_hidden, stream)

    def phase_names(self):
        """Names of the launch groups of a call, in the order their phase events are recorded."""
        groups, chunks = npd_phase_count(self.args)
        names = ["forward_tiles", "merge"]
        for _ in range(chunks):
            names += ["gradient_tiles", "backward_gemms"]
        names += ["dhidden_convert"] * (groups - len(names))
        return names

    def new_phase_events(self, stream=None):
        """groups + 1 timing events, each recorded once so that it owns a CUDA handle."""
        evs = [torch.cuda.Event(enable_timing=True) for _ in range(len(self.phase_names()) + 1)]
        s = torch.cuda.current_stream() if stream is None else stream
        for e in evs:
            e.record(s)
        return evs

    def run_recording(self, evs, stream=None):
        """One step with the library's phase events attached; only enqueues.  The join (norm) runs before the
        first event and after the last."""
        arr = (C.c_void_p * len(evs))(*[e.cuda_event for e in evs])
        a = npd_kd_args.from_buffer_copy(self.args)
        a.phase_events = C.cast(arr, C.POINTER(C.c_void_p))
        a.n_phase_events = len(evs)
        self._run(a, stream)

    def run_with_phase_times(self, stream=None):
        """One step with the library's phase events attached.  Returns a list of
        (group name, milliseconds); synchronises."""
        names = self.phase_names()
        evs = self.new_phase_events(stream)
        self.run_recording(evs, stream)
        torch.cuda.synchronize()
        return [(names[i], evs[i].elapsed_time(evs[i + 1])) for i in range(len(names))]

    def status(self, stream=None) -> int:
        return npd_last_status(self._ws_view, stream)
