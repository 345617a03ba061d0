"""Argument checks of npd_linear_fwd / npd_linear_bwd: found on the host before any CUDA call.  No GPU needed;
the addresses are never dereferenced."""

import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2605_05940_b200 import binding as B
from paper_2605_05940_b200 import build as npd_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BASE = 1 << 20
M, N, K = 5, 24, 40


@pytest.fixture(scope="module", autouse=True)
def _built():
    npd_build.build()


def _args(**kw):
    a = B.npd_linear_args()
    a.size, a.M, a.N, a.K, a.activation = C.sizeof(a), M, N, K, B.NPD_ACT_GELU
    a.x, a.weight, a.bias, a.residual, a.y, a.preact, a.dy, a.dx, a.dw, a.dbias = (BASE * i for i in range(1, 11))
    a.ldx = a.ldw = a.lddx = a.lddw = K
    a.ldr = a.ldy = a.ldz = a.lddy = N
    a.workspace, a.workspace_bytes = 64 * BASE, 1 << 40
    for k, v in kw.items():
        setattr(a, k, v)
    return C.byref(a)


def _fwd(**kw):
    return B.lib().npd_linear_fwd(_args(**kw), None)


def _bwd(**kw):
    return B.lib().npd_linear_bwd(_args(**kw), None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up")
def test_valid_arguments_reach_the_device():
    for kw in ({}, dict(y=4 * BASE), dict(bias=None), dict(residual=None), dict(preact=None), dict(bias=3 * BASE + 2),
               dict(y_dtype=1), dict(y_dtype=1, y=4 * BASE)):
        assert _fwd(**kw) == B.NPD_ECUDA, kw
    for kw in ({}, dict(dx=None), dict(dw=None, x=None), dict(dbias=None), dict(dx=None, dw=None), dict(activation=0, preact=None),
               dict(dw_dtype=1, flags=1)):
        assert _bwd(**kw) == B.NPD_ECUDA, kw
        assert B.lib().npd_linear_workspace_bytes(_args(**kw), C.byref(C.c_size_t(0))) == B.NPD_ECUDA


COMMON = [
    (dict(size=0), B.NPD_EINVAL), (dict(M=0), B.NPD_EINVAL), (dict(N=0), B.NPD_EINVAL), (dict(K=-1), B.NPD_EINVAL),
    (dict(M=(1 << 30) + 1), B.NPD_ESHAPE), (dict(M=1 << 29, N=1 << 29, ldy=1 << 29), B.NPD_ESHAPE),
    (dict(activation=5), B.NPD_EINVAL), (dict(activation=-1), B.NPD_EINVAL), (dict(bias_dtype=2), B.NPD_EINVAL),
    (dict(y_dtype=3), B.NPD_EINVAL), (dict(dw_dtype=-1), B.NPD_EINVAL), (dict(flags=2), B.NPD_EINVAL),
    (dict(flags=B.NPD_LINEAR_ACCUMULATE_DW), B.NPD_EINVAL), (dict(weight=None), B.NPD_EINVAL),
    (dict(ldw=32), B.NPD_ESHAPE), (dict(ldw=44), B.NPD_EALIGN), (dict(weight=2 * BASE + 8), B.NPD_EALIGN),
]


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(x=None), B.NPD_EINVAL), (dict(y=None), B.NPD_EINVAL), (dict(ldy=16), B.NPD_ESHAPE), (dict(ldz=28), B.NPD_EALIGN),
    (dict(bias=3 * BASE + 2, bias_dtype=1), B.NPD_EALIGN), (dict(status=11 * BASE + 2), B.NPD_EALIGN),
    (dict(y=BASE), B.NPD_EINVAL), (dict(y=2 * BASE), B.NPD_EINVAL), (dict(y=4 * BASE + 2 * N), B.NPD_EINVAL),
    (dict(preact=5 * BASE), B.NPD_EINVAL), (dict(preact=4 * BASE), B.NPD_EINVAL), (dict(preact=BASE), B.NPD_EINVAL),
    (dict(y=3 * BASE), B.NPD_EINVAL),
])
def test_forward_refusals(kw, code):
    assert _fwd(**kw) == code


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(dy=None), B.NPD_EINVAL), (dict(dx=None, dw=None, dbias=None), B.NPD_EINVAL), (dict(preact=None), B.NPD_EINVAL),
    (dict(x=None), B.NPD_EINVAL), (dict(lddx=16), B.NPD_ESHAPE), (dict(x=BASE + 2), B.NPD_EALIGN),
    (dict(dbias=10 * BASE + 1), B.NPD_EALIGN), (dict(dx=BASE), B.NPD_EINVAL), (dict(dx=7 * BASE), B.NPD_EINVAL),
    (dict(dw=2 * BASE), B.NPD_EINVAL), (dict(dx=9 * BASE), B.NPD_EINVAL), (dict(dbias=9 * BASE), B.NPD_EINVAL),
    (dict(dx=6 * BASE), B.NPD_EINVAL),
])
def test_backward_refusals(kw, code):
    assert _bwd(**kw) == code


def test_null_arguments():
    assert B.lib().npd_linear_fwd(None, None) == B.NPD_EINVAL and B.lib().npd_linear_bwd(None, None) == B.NPD_EINVAL
    assert B.lib().npd_linear_workspace_bytes(_args(), None) == B.NPD_EINVAL
    for f in (lambda: B.npd_linear_fwd(None, None), lambda: B.npd_linear_bwd(None, None, None),
              lambda: B.npd_linear_fwd(torch.zeros((2, 8), dtype=torch.bfloat16), torch.zeros((2, 8), dtype=torch.bfloat16))):
        with pytest.raises(B.NpdError):
            f()


def test_struct_layout_matches_the_header(tmp_path):
    fields = [f[0] for f in B.npd_linear_args._fields_]
    src = "#include <stdio.h>\n#include <stddef.h>\n#include \"npd.h\"\nint main(void){printf(\"%zu\", sizeof(npd_linear_args));" + \
        "".join(f'printf(" %zu", offsetof(npd_linear_args, {f}));' for f in fields) + "return 0;}"
    c = tmp_path / "t.c"
    c.write_text(src)
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(c), "-o", str(tmp_path / "t")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(B.npd_linear_args)] + [getattr(B.npd_linear_args, f).offset for f in fields]


@pytest.mark.parametrize("kw", [dict(M=(1 << 23) + 1, N=1 << 23), dict(N=1 << 30, K=(1 << 16) + 1), dict(M=1 << 30, K=(1 << 16) + 1)])
def test_products_beyond_the_limit_are_refused(kw):
    assert B.lib().npd_linear_workspace_bytes(_args(**kw), C.byref(C.c_size_t(0))) == B.NPD_ESHAPE


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up")
@pytest.mark.parametrize("kw", [dict(M=1 << 23, N=1 << 23), dict(M=(1 << 23) + 1, N=(1 << 23) - 1), dict(N=1 << 30, K=1 << 16)])
def test_products_up_to_the_limit_pass(kw):
    # whole tiles beyond a border do not count against it
    assert B.lib().npd_linear_workspace_bytes(_args(**kw), C.byref(C.c_size_t(0))) == B.NPD_ECUDA
