"""Argument checks of npd_ce_fwd_bwd: found on the host before any CUDA call.  No GPU needed; the
addresses are never dereferenced."""

import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2605_05940_b200 import binding as B
from paper_2605_05940_b200 import build as npd_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BASE = 1 << 20
T, D, V = 5, 64, 40


@pytest.fixture(scope="module", autouse=True)
def _built():
    npd_build.build()


def _args(**kw):
    a = B.npd_ce_args()
    a.size, a.T, a.d, a.V, a.temperature, a.grad_scale = C.sizeof(a), T, D, V, 1.0, 1.0
    a.hidden, a.weight, a.labels, a.nll, a.lse, a.d_hidden, a.d_weight = (BASE * i for i in range(1, 8))
    a.ldh = a.ldw = a.ld_dh = a.ld_dw = D
    a.workspace, a.workspace_bytes = 64 * BASE, 1 << 40
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _run(**kw):
    return B.lib().npd_ce_fwd_bwd(C.byref(_args(**kw)), None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up")
def test_valid_arguments_reach_the_device():
    for kw in ({}, dict(d_hidden=None), dict(d_weight=None), dict(d_hidden=None, d_weight=None), dict(lse=None),
               dict(loss_mask=9 * BASE + 1), dict(d_weight_dtype=1, flags=3)):
        assert _run(**kw) == B.NPD_ECUDA, kw
        n = C.c_size_t(0)
        assert B.lib().npd_ce_workspace_bytes(C.byref(_args(**kw)), C.byref(n)) == B.NPD_ECUDA


@pytest.mark.parametrize("kw,code", [
    (dict(size=0), B.NPD_EINVAL), (dict(T=0), B.NPD_EINVAL), (dict(V=0), B.NPD_EINVAL), (dict(d=0), B.NPD_EINVAL),
    (dict(d=96), B.NPD_ESHAPE), (dict(T=(1 << 30) + 1), B.NPD_ESHAPE), (dict(V=(1 << 30) + 1), B.NPD_ESHAPE),
    (dict(temperature=0.0), B.NPD_EINVAL), (dict(temperature=float("nan")), B.NPD_EINVAL),
    (dict(grad_scale=float("inf")), B.NPD_EINVAL), (dict(d_weight_dtype=2), B.NPD_EINVAL),
    (dict(flags=4), B.NPD_EINVAL), (dict(flags=B.NPD_CE_ACCUMULATE_DW), B.NPD_EINVAL),
    (dict(grad_chunk_cols=-1), B.NPD_EINVAL), (dict(hidden=None), B.NPD_EINVAL), (dict(weight=None), B.NPD_EINVAL),
    (dict(labels=None), B.NPD_EINVAL), (dict(nll=None), B.NPD_EINVAL), (dict(ldh=32), B.NPD_ESHAPE),
    (dict(ld_dw=56), B.NPD_ESHAPE), (dict(ldw=68), B.NPD_EALIGN), (dict(hidden=BASE + 8), B.NPD_EALIGN),
    (dict(labels=3 * BASE + 2), B.NPD_EALIGN), (dict(token_weight=9 * BASE + 1), B.NPD_EALIGN),
    (dict(d_hidden=BASE), B.NPD_EINVAL), (dict(d_weight=2 * BASE), B.NPD_EINVAL), (dict(lse=4 * BASE), B.NPD_EINVAL),
    (dict(d_weight=6 * BASE + 2 * D), B.NPD_EINVAL),
])
def test_refusals(kw, code):
    assert _run(**kw) == code


def test_null_arguments():
    assert B.lib().npd_ce_fwd_bwd(None, None) == B.NPD_EINVAL
    assert B.lib().npd_ce_workspace_bytes(None, C.byref(C.c_size_t())) == B.NPD_EINVAL
    assert B.lib().npd_ce_workspace_bytes(C.byref(_args()), None) == B.NPD_EINVAL
    with pytest.raises(B.NpdError):
        B.npd_cross_entropy(torch.zeros((2, 64), dtype=torch.bfloat16), None, None)


def test_struct_layout_matches_the_header(tmp_path):
    fields = [f[0] for f in B.npd_ce_args._fields_]
    src = "#include <stdio.h>\n#include <stddef.h>\n#include \"npd.h\"\nint main(void){printf(\"%zu\", sizeof(npd_ce_args));" + \
        "".join(f'printf(" %zu", offsetof(npd_ce_args, {f}));' for f in fields) + "return 0;}"
    c = tmp_path / "t.c"
    c.write_text(src)
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(c), "-o", str(tmp_path / "t")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(B.npd_ce_args)] + [getattr(B.npd_ce_args, f).offset for f in fields]


def _wide(d, **kw):
    return dict(dict(d=d, ldh=d, ldw=d, ld_dh=d, ld_dw=d), **kw)


@pytest.mark.parametrize("kw", [
    # from d = 2^27 on the bytes of eight tokens pass 32 bits; at 2^28 they would wrap to none at all
    _wide(1 << 27), _wide(1 << 28), _wide((1 << 28) + 64, T=1, V=2, d_hidden=None, d_weight=None), _wide(1 << 30),
    _wide((1 << 26) + 64), _wide(1 << 26, V=(1 << 20) + 1), _wide(1 << 26, T=(1 << 20) + 1),
    dict(T=(1 << 23) + 1, V=1 << 23), dict(T=1 << 30, V=(1 << 16) + 1),
])
def test_extents_beyond_the_limits_are_refused(kw):
    assert _run(**kw) == B.NPD_ESHAPE
    n = C.c_size_t(0)
    assert B.lib().npd_ce_workspace_bytes(C.byref(_args(**kw)), C.byref(n)) == B.NPD_ESHAPE


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up")
@pytest.mark.parametrize("kw", [dict(T=1 << 23, V=1 << 23), dict(T=1 << 30, V=1 << 16), dict(T=(1 << 23) - 1, V=(1 << 23) + 1),
                                _wide(1 << 26)])
def test_extents_up_to_the_limits_pass(kw):
    n = C.c_size_t(0)
    assert B.lib().npd_ce_workspace_bytes(C.byref(_args(**kw)), C.byref(n)) == B.NPD_ECUDA
