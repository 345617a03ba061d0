"""Argument checks of npd_norm_fwd / npd_norm_bwd: refusals are found on the host before any CUDA call.
No GPU needed; the addresses are never dereferenced."""

import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2605_05940_b200 import binding as B
from paper_2605_05940_b200 import build as npd_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
T, D = 4, 40
BASE = 1 << 20          # addresses of the operands: BASE * n


@pytest.fixture(scope="module", autouse=True)
def _built():
    npd_build.build()


def _fwd(**kw):
    a = B.npd_norm_args()
    a.size, a.T, a.d, a.eps, a.residual_scale, a.branch_scale = C.sizeof(a), T, D, 1e-6, 1.0, 1.0
    a.x, a.residual, a.h, a.y = BASE, 2 * BASE, 3 * BASE, 4 * BASE
    a.ldx = a.ldr = a.ldh = a.ldy = D
    for k, v in kw.items():
        setattr(a, k, v)
    return B.lib().npd_norm_fwd(C.byref(a), None)


def _bwd(**kw):
    a = B.npd_norm_args()
    a.size, a.T, a.d, a.eps, a.residual_scale, a.branch_scale = C.sizeof(a), T, D, 1e-6, 1.0, 1.0
    a.x, a.h, a.dy, a.dh, a.dx, a.dresidual = (BASE * i for i in range(1, 7))
    a.ldx = a.ldh = a.lddy = a.lddh = a.lddx = a.lddr = D
    for k, v in kw.items():
        setattr(a, k, v)
    return B.lib().npd_norm_bwd(C.byref(a), None)


# what a call gets that passes every check: the device's answer, on a box without one NPD_ECUDA
@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up")
@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_valid_arguments_reach_the_device(call):
    assert call() == B.NPD_ECUDA


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up")
def test_results_may_take_an_operands_place():
    for kw in (dict(h=2 * BASE), dict(h=BASE), dict(y=BASE), dict(y=2 * BASE), dict(h=None), dict(y=None),
               dict(x=None), dict(residual=None), dict(gate=7 * BASE), dict(gate=7 * BASE, ldg=D),
               dict(h=BASE * 3, y=BASE * 3 + 2 * D, ldh=2 * D, ldy=2 * D)):          # two halves of one buffer
        assert _fwd(**kw) == B.NPD_ECUDA, kw
    for kw in (dict(dx=BASE), dict(dx=3 * BASE), dict(dresidual=4 * BASE), dict(dresidual=2 * BASE),
               dict(dy=None, h=None), dict(dh=None), dict(x=None, dx=None),
               dict(gate=8 * BASE, ldg=D, d_gate=8 * BASE, lddg=D)):
        assert _bwd(**kw) == B.NPD_ECUDA, kw


@pytest.mark.parametrize("kw,code", [
    (dict(size=8), B.NPD_EINVAL), (dict(T=0), B.NPD_EINVAL), (dict(d=0), B.NPD_EINVAL), (dict(d=16385), B.NPD_ESHAPE),
    (dict(stream_dtype=2), B.NPD_EINVAL), (dict(weight_dtype=-1), B.NPD_EINVAL), (dict(flags=2), B.NPD_EINVAL),
    (dict(eps=-1.0), B.NPD_EINVAL), (dict(eps=float("nan")), B.NPD_EINVAL),
    (dict(branch_scale=float("inf")), B.NPD_EINVAL),
    (dict(x=BASE + 2), B.NPD_EALIGN), (dict(ldx=D + 1), B.NPD_EALIGN), (dict(ldx=D - 8), B.NPD_ESHAPE),
    (dict(ldr=0), B.NPD_ESHAPE), (dict(x=None, residual=None), B.NPD_EINVAL), (dict(h=None, y=None), B.NPD_EINVAL),
    (dict(x=None, flags=B.NPD_NORM_POST), B.NPD_EINVAL), (dict(x=None, gate=8 * BASE), B.NPD_EINVAL),
    (dict(pre_weight=8 * BASE + 1), B.NPD_EALIGN), (dict(post_weight=8 * BASE + 2, weight_dtype=1), B.NPD_EALIGN),
    (dict(h=3 * BASE, y=3 * BASE), B.NPD_EINVAL), (dict(h=BASE + 2 * D), B.NPD_EINVAL),        # partial overlap
    (dict(h=2 * BASE, stream_dtype=1, y=2 * BASE), B.NPD_EINVAL),
    (dict(gate=4 * BASE), B.NPD_EINVAL), (dict(pre_weight=4 * BASE), B.NPD_EINVAL),
    (dict(gate=7 * BASE, ldg=8), B.NPD_ESHAPE),
])
def test_forward_refusals(kw, code):
    assert _fwd(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None, dh=None), B.NPD_EINVAL), (dict(h=None), B.NPD_EINVAL),
    (dict(dx=None, dresidual=None), B.NPD_EINVAL), (dict(d_post_weight=9 * BASE), B.NPD_EINVAL),
    (dict(dy=None, d_pre_weight=9 * BASE), B.NPD_EINVAL), (dict(d_gate=9 * BASE), B.NPD_EINVAL),
    (dict(gate=8 * BASE, ldg=D, d_gate=9 * BASE, lddg=8), B.NPD_ESHAPE),
    (dict(gate=8 * BASE, ldg=D, d_gate=9 * BASE + 2, lddg=D), B.NPD_EALIGN),
    (dict(gate=8 * BASE, d_gate=8 * BASE), B.NPD_EINVAL),            # a shared gate's gradient is fp32
    (dict(d_pre_weight=9 * BASE + 2), B.NPD_EALIGN),
    (dict(dx=5 * BASE, dresidual=5 * BASE), B.NPD_EINVAL), (dict(dx=3 * BASE + 2 * D), B.NPD_EINVAL),
    (dict(dresidual=4 * BASE, stream_dtype=1, dx=4 * BASE), B.NPD_EINVAL),
    (dict(pre_weight=6 * BASE), B.NPD_EINVAL),
])
def test_backward_refusals(kw, code):
    assert _bwd(**kw) == code


def test_struct_layout_matches_the_header(tmp_path):
    fields = [f[0] for f in B.npd_norm_args._fields_]
    src = "#include <stdio.h>\n#include <stddef.h>\n#include \"npd.h\"\nint main(void){printf(\"%zu\", sizeof(npd_norm_args));" + \
        "".join(f'printf(" %zu", offsetof(npd_norm_args, {f}));' for f in fields) + "return 0;}"
    c = tmp_path / "t.c"
    c.write_text(src)
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(c), "-o", str(tmp_path / "t")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(B.npd_norm_args)] + [getattr(B.npd_norm_args, f).offset for f in fields]


def test_tensors_of_the_wrong_kind_are_refused():
    x = torch.zeros((4, 8), dtype=torch.bfloat16)
    with pytest.raises(B.NpdError):
        B.npd_norm_fwd(x)                    # not on a GPU
    with pytest.raises(B.NpdError):
        B.npd_norm_fwd(None)
    with pytest.raises(B.NpdError):
        B.npd_norm_bwd(None, None)
